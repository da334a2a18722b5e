// Routing: a gate's scores choose members for each row, and weigh them.
//   s = softmax(x) or sigmoid(x) over the members; a member ranks by c = s + bias as 64 bits give it, or by x where there are neither bias nor groups (s rises
//   with x)
//   groups of neighbouring members rank by the sum of their one or two best c; members of the best groups stay
//   the k best c are chosen, the lowest member on equal ones; weight = scale s, or scale s / (sum of the chosen s)
// x of minus infinity or NaN: not a member of this row.
//
// A wavefront takes a row, up to eight neighbouring members a lane.  Bound by vector instructions, k choices one after the other (a maximum over
// the lanes is six shifted maxima): 32 768 rows of 256 bf16 members, k = 8, 22 us with the counts, 276 vector instructions a row, where the bytes
// take 4 us; with a bias 37 us (softmax) to 42 (sigmoid), in eight groups 45 to 49, both 52 to 57, without the counts.  The gradient 10 us.  With a bias or groups the 64
// registers that leave room for eight wavefronts are too few: 3 to 5 are spilled at 128 members, 15 to 20 at 256.
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

enum { SCORE_SOFTMAX = 0, SCORE_SIGMOID = 1 };
// Rows at a time of a workgroup.  A workgroup adds what its rows chose to `load` once for each member, and these additions meet on few addresses: with
// 4 rows and 2 048 workgroups they took 30 us of 55 (32 768 rows of 256 members).
template <int PER> constexpr int ROUTE_WAVES = PER == 8 ? 8 : 16;

// Over the 64 lanes in 64 bits.
__device__ __forceinline__ double lanes_max(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float of_lane(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }
__device__ __forceinline__ double of_lane(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = __builtin_amdgcn_readlane((uint32_t)b, lane), high = __builtin_amdgcn_readlane((uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ float exp_r(float v) { return __builtin_amdgcn_exp2f(v * LOG2E); }      // for v <= 0, as rows.h says
__device__ __forceinline__ double exp_r(double v) { return exp(v); }
__device__ __forceinline__ float over(float x, float y) { return x * __builtin_amdgcn_rcpf(y); }
__device__ __forceinline__ double over(double x, double y) { return x / y; }

// Member lane * PER + j of a row in v[j], `otherwise` behind the last.
template <class T, int PER>
__device__ __forceinline__ void load_members(const T* p, int members, int lane, T otherwise, T (&v)[PER]) {
    const int first = lane * PER;
    if (first + PER <= members) load_few(p + first, v);
    else
#pragma unroll
        for (int j = 0; j < PER; j++) v[j] = first + j < members ? p[first + j] : otherwise;
}

// A gate's value; not a member: minus infinity.
__device__ __forceinline__ float gate_value(float x) { return x > NONE ? fminf(x, -LOWEST) : NONE; }
template <class R>
__device__ __forceinline__ R sigmoid_of(R x) {
    const R e = exp_r(x >= 0 ? -x : x);
    return over(x >= 0 ? 1 : e, 1 + e);
}
// Logarithm of the score up to a constant of the row.
__device__ __forceinline__ float log_score(int score, float x) {
    if (score == SCORE_SOFTMAX) return x;
    return fminf(x, 0.f) - log1pf(expf(-fabsf(x)));
}

// Maximum and sum of e^(x - maximum) over the members of a row.
template <class R, int PER>
__device__ __forceinline__ void softmax_of(const R (&x)[PER], R& m, R& sum) {
    m = x[0];
#pragma unroll
    for (int j = 1; j < PER; j++) m = x[j] > m ? x[j] : m;
    m = lanes_max(m);
    sum = 0;
    if (!(m > NONE)) return;
#pragma unroll
    for (int j = 0; j < PER; j++) sum += exp_r(x[j] - m);
    sum = lanes_sum(sum);
}

// What a row's choice goes by.
struct Rule {
    const float* bias;
    int members, k, score, groups, groups_kept, group_best;
};

// What members rank by, in c (minus infinity: not there), with a bias or in groups; x as gate_value gives it, member lane * PER + j in x[j].
template <class R, int PER>
__device__ __forceinline__ void member_ranks(const Rule& a, int lane, const float (&x)[PER], R (&c)[PER], R& most) {
    R v[PER], m = 0, sum = 1;
#pragma unroll
    for (int j = 0; j < PER; j++) v[j] = x[j];
    if (a.score == SCORE_SOFTMAX) softmax_of<R, PER>(v, m, sum);
    most = 0;
    float bias[PER];
#pragma unroll
    for (int j = 0; j < PER; j++) bias[j] = 0.f;
    if (a.bias) load_members(a.bias, a.members, lane, 0.f, bias);
    const R inverse = over((R)1, sum);
#pragma unroll
    for (int j = 0; j < PER; j++) {
        const R s = a.score == SCORE_SOFTMAX ? exp_r(v[j] - m) * inverse : sigmoid_of(v[j]);
        c[j] = s + (R)bias[j];
        if (!(x[j] > NONE) || !(c[j] > (R)NONE)) c[j] = (R)NONE;
        else most = fmax(most, s + fabs((R)bias[j]));
    }
    most = lanes_max(most);
}

// Takes members of the groups that do not stay out of c.  `ranks`: PER * 64 values of LDS.  Lanes share a group's members; the least difference
// between a group that stays and one that does not is returned.
template <class R, int PER>
__device__ __forceinline__ R drop_groups(const Rule& a, int lane, R (&c)[PER], R* ranks) {
    const R none = (R)NONE;
    const int size = a.members / a.groups;
    const int each = 64 >> (32 - __clz(a.groups - 1));           // lanes of a group (two groups at least)
    const int group = lane / each;
#pragma unroll
    for (int j = 0; j < PER; j++) ranks[lane * PER + j] = c[j];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    R first = none, second = none;
    auto take = [&](R v) {
        second = fmax(second, fmin(first, v));
        first = fmax(first, v);
    };
    if (group < a.groups)
        for (int i = lane % each; i < size; i += each) take(ranks[group * size + i]);
    for (int o = 1; o < each; o <<= 1) {
        const R f = __shfl_xor(first, o, 64), s = __shfl_xor(second, o, 64);
        take(f);
        second = fmax(second, s);
    }
    const R rank = a.group_best == 2 && second > none ? first + second : first;
    int better = 0;
    for (int g = 0; g < a.groups; g++) {
        const R other = of_lane(rank, g * each);
        better += other > rank || (other == rank && g < group);
    }
    const bool stays = group < a.groups && better < a.groups_kept;
    const unsigned long long kept = __ballot(stays);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint32_t inverse = ((1u << 20) + size - 1) / size;     // members below 512: e * inverse >> 20 is e / size
#pragma unroll
    for (int j = 0; j < PER; j++) {
        const int of = (int)((uint32_t)(lane * PER + j) * inverse >> 20);
        if (lane * PER + j < a.members && !(kept >> (of * each) & 1)) c[j] = none;
    }
    if (a.groups_kept == a.groups) return (R)__builtin_inf();
    const R in = -lanes_max(stays ? -rank : none), out = lanes_max(stays || group >= a.groups ? none : rank);
    return out > none ? in - out : (R)__builtin_inf();
}

// The k best of c, the i-th in lane i, -1 behind the last.  gap: the least difference between one and the next, the best that is left among
// them.  Members of equal rank come in no order, with a gap of 0.
template <int PER>
__device__ __forceinline__ int best_members(int k, int lane, const float (&c)[PER], float& gap) {
    // the lane's ranks in falling order, as whole numbers (0: not there), and the members' numbers in the lane with them
    uint32_t key[PER], number[PER];
#pragma unroll
    for (int j = 0; j < PER; j++) {
        key[j] = c[j] > NONE ? ordered(c[j]) : 0u;
        number[j] = j;
    }
#pragma unroll
    for (int size = 2; size <= PER; size *= 2)
#pragma unroll
        for (int step = size / 2; step > 0; step /= 2)
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int o = i ^ step;
                if (o < i) continue;
                const bool falling = (i & size) == 0 || size == PER;
                const uint32_t swap = (falling ? key[i] < key[o] : key[o] < key[i]) ? ~0u : 0u;
                const uint32_t keys = (key[i] ^ key[o]) & swap, numbers = (number[i] ^ number[o]) & swap;
                key[i] ^= keys; key[o] ^= keys; number[i] ^= numbers; number[o] ^= numbers;
            }
    int mine = -1;
    float before = __builtin_inff();
    gap = __builtin_inff();
    for (int i = 0; i <= k; i++) {
        const uint32_t most = lanes_max(key[0]);
        if (most == 0) break;
        const float best = unordered(most);
        if (i > 0) gap = fminf(gap, before == best ? 0.f : before - best);
        before = best;
        if (i == k) break;
        const int owner = __builtin_ctzll(__ballot(key[0] == most)), at = owner * PER + __builtin_amdgcn_readlane(number[0], owner);
        if (lane == i) mine = at;
        const uint32_t taken = lane == owner ? ~0u : 0u;
#pragma unroll
        for (int j = 0; j + 1 < PER; j++) {
            key[j] = (key[j + 1] & taken) | (key[j] & ~taken);
            number[j] = (number[j + 1] & taken) | (number[j] & ~taken);
        }
        key[PER - 1] &= ~taken;
    }
    return mine;
}

// The same with the lowest member first among equal ranks.
template <class R, int PER>
__device__ __forceinline__ int best_in_order(int k, int lane, R (&c)[PER]) {
    int mine = -1;
    for (int i = 0; i < k; i++) {
        R best = c[0];
#pragma unroll
        for (int j = 1; j < PER; j++) best = fmax(best, c[j]);
        best = lanes_max(best);
        if (!(best > (R)NONE)) break;
        int own = -1;
#pragma unroll
        for (int j = PER - 1; j >= 0; j--) own = c[j] == best ? j : own;
        const int owner = __builtin_ctzll(__ballot(own >= 0)), at = owner * PER + __builtin_amdgcn_readlane(own, owner);
#pragma unroll
        for (int j = 0; j < PER; j++) c[j] = lane == owner && own == j ? (R)NONE : c[j];
        if (lane == i) mine = at;
    }
    return mine;
}

// The same in 64 bits, for rows in which 32 do not tell two ranks apart.
template <class T, int PER>
__device__ __attribute__((noinline)) int choose_exactly(const Rule a, const T* gates, double* ranks) {
    const int lane = threadIdx.x & 63;
    T raw[PER];
    float x[PER];
    double c[PER], most;
    load_members(gates, a.members, lane, (T)NONE, raw);
#pragma unroll
    for (int j = 0; j < PER; j++) x[j] = gate_value(up(raw[j]));
    member_ranks<double, PER>(a, lane, x, c, most);
    if (a.groups > 1) drop_groups<double, PER>(a, lane, c, ranks);
    return best_in_order<double, PER>(a.k, lane, c);
}

__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(__bf16 v) { return __builtin_bit_cast(uint16_t, v); }
__device__ __forceinline__ uint32_t bits_of(_Float16 v) { return __builtin_bit_cast(uint16_t, v); }

// Gate values of 16 bits by themselves: value and member in one key, no two alike and 0 for what is not there.
template <int PER>
__device__ __forceinline__ int best_of_keys(int k, int lane, uint32_t (&key)[PER]) {
    int mine = -1;
#pragma unroll
    for (int size = 2; size <= PER; size *= 2)
#pragma unroll
        for (int step = size / 2; step > 0; step /= 2)
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int o = i ^ step;
                if (o < i) continue;
                const uint32_t low = min(key[i], key[o]), high = max(key[i], key[o]);
                const bool falling = (i & size) == 0 || size == PER;
                key[i] = falling ? high : low;
                key[o] = falling ? low : high;
            }
    for (int i = 0; i < k; i++) {
        const uint32_t best = lanes_max(key[0]);
        if (best == 0) break;
        if (lane == i) mine = 0xFFFF - (int)(best & 0xFFFFu);
        const uint32_t taken = key[0] == best ? ~0u : 0u;
#pragma unroll
        for (int j = 0; j + 1 < PER; j++) key[j] = (key[j + 1] & taken) | (key[j] & ~taken);
        key[PER - 1] &= ~taken;
    }
    return mine;
}

// By the gate's values themselves, those of them whose x is not minus infinity.
template <class T, int PER>
__device__ __forceinline__ int best_by_value(int k, int lane, const T (&raw)[PER], const float (&x)[PER]) {
    if constexpr (sizeof(T) == 2) {
        uint32_t key[PER];
#pragma unroll
        for (int j = 0; j < PER; j++) {
            uint32_t b = bits_of(raw[j]) << 16;
            b = b == 0x80000000u ? 0u : b;                       // both zeros are one
            b ^= (uint32_t)((int32_t)b >> 31) | 0x80000000u;
            key[j] = x[j] > NONE ? (b & 0xFFFF0000u) | (uint32_t)(0xFFFF - (lane * PER + j)) : 0u;
        }
        return best_of_keys<PER>(k, lane, key);
    } else {
        float c[PER];
#pragma unroll
        for (int j = 0; j < PER; j++) c[j] = x[j];
        return best_in_order<float, PER>(k, lane, c);
    }
}

// BY_VALUE: members rank by the gate's values themselves (no bias, no groups).
template <class T, int PER, bool BY_VALUE>
__global__ __launch_bounds__(64 * ROUTE_WAVES<PER>, PER <= 4 ? 8 : 4) void route_kernel(const RouteArgs a) {
    constexpr int WAVES = ROUTE_WAVES<PER>;
    __shared__ int counts[PER * 64];
    __shared__ double ranks[BY_VALUE ? 1 : WAVES][PER * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), E = a.members;
    const Rule rule{a.bias, a.members, a.k, a.score, a.groups, a.groups_kept, a.group_best};
    if (a.load) {
        for (int e = threadIdx.x; e < E; e += 64 * WAVES) counts[e] = 0;
        __syncthreads();
    }
    const int64_t first = (int64_t)blockIdx.x * WAVES + wave, step = (int64_t)gridDim.x * WAVES;
    T next[PER];
    if (first < a.n) load_members((const T*)a.gates + first * a.ld, E, lane, (T)NONE, next);
    for (int64_t row = first; row < a.n; row += step) {
        const T* const gates = (const T*)a.gates + row * a.ld;
        T raw[PER];
        float x[PER];
#pragma unroll
        for (int j = 0; j < PER; j++) {
            raw[j] = next[j];
            x[j] = gate_value(up(raw[j]));
        }
        if (row + step < a.n) load_members(gates + step * a.ld, E, lane, (T)NONE, next);
        int mine;
        bool told = true;
        if (!BY_VALUE) {
            float c[PER], most, gap, apart = __builtin_inff();
            member_ranks<float, PER>(rule, lane, x, c, most);
            if (a.groups > 1) apart = drop_groups<float, PER>(rule, lane, c, (float*)ranks[wave]);
            // A score s = e^d (/ sum) is off by some 20 units of 2^-24 of itself and 2.5 |d| more: d, its product with log2 e and the constant are rounded at their
            // own sizes.  |d| is -ln s at most, and s (1 - (ln s) / 8) rises with s, so that the largest s + |bias| bounds it for all members.
            const float slack = most * fmaf(-__builtin_amdgcn_logf(fmaxf(0x1p-126f, fminf(most, 1.f))), 0.0867f, 1.06f);
            // 256 units between the ranks of two groups, sums of two scores each, 64 between those of two members
            told = apart > fmaf(slack, 0x1p-16f, 0x1p-120f);
            if (a.bias) {
                mine = best_members<PER>(a.k, lane, c, gap);
                told = told && gap > fmaf(slack, 0x1p-18f, 0x1p-120f);
            } else {
                // Members of the groups that stay, by value: their scores rise with it.  Scores of different values are different in 64 bits too, but for tiny ones
                // (0 in 32 bits), values next to 0 (of 2^-18 and more neighbours lie 2^-41 apart, beside a maximum of 105 at most) and sigmoids next to 1 (beyond 20
                // neighbours differ by less than 16 units).  Equal scores are ties, which 64 bits settle: rows with two such values at least.
                uint32_t score = ~0u, near = ~0u;                // the least score, and the least |x| but 0 (less one), as whole numbers
                float far = NONE;
#pragma unroll
                for (int j = 0; j < PER; j++) {
                    x[j] = c[j] > NONE ? x[j] : NONE;
                    score = min(score, __float_as_uint(c[j]));
                    near = min(near, (__float_as_uint(x[j]) & 0x7FFFFFFFu) - 1u);
                    far = fmaxf(far, x[j]);
                }
                told = told && __ballot(score == 0u) == 0;
                const bool large = a.score == SCORE_SIGMOID && far > 20.f;
                if (__ballot(near < __float_as_uint(0x1p-18f) - 1u || large) != 0) {
                    int near_zero = 0, near_one = 0;
#pragma unroll
                    for (int j = 0; j < PER; j++) {
                        near_zero += __popcll(__ballot(fabsf(x[j]) < 0x1p-18f));
                        near_one += __popcll(__ballot(large && x[j] > 20.f));
                    }
                    told = told && near_zero < 2 && near_one < 2;
                }
            }
        }
        if (BY_VALUE || !a.bias) mine = best_by_value<T, PER>(a.k, lane, raw, x);
        if (!told) mine = choose_exactly<T, PER>(rule, gates, ranks[wave]);
        const float own = mine >= 0 ? gate_value(up(gates[mine])) : NONE;
        float weight;
        if (a.renormalise) {
            const float l = mine >= 0 ? log_score(a.score, own) : NONE, top = lanes_max(l);
            const float e = mine >= 0 ? expf(l - top) : 0.f, sum = lanes_sum(e);
            weight = mine >= 0 ? e / sum : 0.f;
        } else if (a.score == SCORE_SIGMOID) {
            weight = mine >= 0 ? sigmoid_of(own) : 0.f;
        } else {
            float m, sum;
#pragma unroll
            for (int j = 0; j < PER; j++) x[j] = gate_value(up(raw[j]));     // of all members, also of groups that do not stay
            softmax_of<float, PER>(x, m, sum);
            weight = mine >= 0 ? expf(own - m) / sum : 0.f;
        }
        if (lane < a.k) {
            a.chosen[row * a.k + lane] = mine;
            a.weights[row * a.k + lane] = weight * a.scale;
            if (a.load && mine >= 0) atomicAdd(&counts[mine], 1);
        }
    }
    if (a.load) {
        __syncthreads();
        for (int e = threadIdx.x; e < E; e += 64 * WAVES)
            if (counts[e]) atomicAdd(&a.load[e], counts[e]);
    }
}

// u_j = scale dL/dw_j.  Renormalised: r = softmax over the chosen of ln s, dL/d(ln s_j) = r_j (u_j - sum r u); softmax: that is dL/dx_j,
// sigmoid: times 1 - s_j.  As they are: softmax dL/dx_e = s_e (u_e - sum u_j s_j), sigmoid dL/dx_j = u_j s_j (1 - s_j).
// The choice itself has no derivative.
template <class T, int PER>
__global__ __launch_bounds__(64 * ROUTE_WAVES<PER>) void route_backward_kernel(const RouteArgs a) {
    constexpr int WAVES = ROUTE_WAVES<PER>;
    __shared__ float parts[WAVES][PER * 64];                     // of the row's members, zeros between rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), E = a.members;
    float* const part = parts[wave];
#pragma unroll
    for (int j = 0; j < PER; j++) part[lane * PER + j] = 0.f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int64_t row = (int64_t)blockIdx.x * WAVES + wave; row < a.n; row += (int64_t)gridDim.x * WAVES) {
        const T* const gates = (const T*)a.gates + row * a.ld;
        int mine = lane < a.k ? a.chosen[row * a.k + lane] : -1;
        if (mine < 0 || mine >= E) mine = -1;
        const float u = mine >= 0 ? a.scale * a.d_weights[row * a.k + lane] : 0.f;
        const float own = mine >= 0 ? gate_value(up(gates[mine])) : NONE;
        if (!(own > NONE)) mine = -1;
        const bool dense = !a.renormalise && a.score == SCORE_SOFTMAX;
        float slot = 0.f, mean = 0.f, m = 0.f, sum = 1.f;
        T raw[PER];
        if (a.renormalise) {
            const float l = mine >= 0 ? log_score(a.score, own) : NONE, top = lanes_max(l);
            const float e = mine >= 0 ? expf(l - top) : 0.f, total = lanes_sum(e);
            const float r = mine >= 0 ? e / total : 0.f;
            slot = r * (u - lanes_sum(r * u));
            if (a.score == SCORE_SIGMOID && mine >= 0) slot *= sigmoid_of(-own);
        } else if (a.score == SCORE_SIGMOID) {
            if (mine >= 0) slot = u * sigmoid_of(own) * sigmoid_of(-own);
        } else {
            float x[PER];
            load_members(gates, E, lane, (T)NONE, raw);
#pragma unroll
            for (int j = 0; j < PER; j++) x[j] = gate_value(up(raw[j]));
            softmax_of<float, PER>(x, m, sum);
            if (mine >= 0) slot = u * (expf(own - m) / sum);
            mean = lanes_sum(slot);
        }
        // to the members through LDS; a member that was chosen twice gets both, in order
        if (mine >= 0) part[mine] = __int_as_float(lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool twice = mine >= 0 && __float_as_int(part[mine]) != lane;
        if (__ballot(twice) == 0) {
            if (mine >= 0) part[mine] = slot;
        } else {
            if (mine >= 0) part[mine] = 0.f;
            for (int i = 0; i < a.k; i++) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (lane == i && mine >= 0) part[mine] += slot;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float d[PER];
        T out[PER];
#pragma unroll
        for (int j = 0; j < PER; j++) d[j] = part[lane * PER + j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (mine >= 0) part[mine] = 0.f;
        if (dense)
#pragma unroll
            for (int j = 0; j < PER; j++) {
                const float x = gate_value(up(raw[j]));
                if (x > NONE) d[j] -= expf(x - m) / sum * mean;
            }
#pragma unroll
        for (int j = 0; j < PER; j++) out[j] = (T)d[j];
        T* const to = (T*)a.d_gates + row * a.ld_d + lane * PER;
        if ((lane + 1) * PER <= E) store_few(to, out);
        else
#pragma unroll
            for (int j = 0; j < PER; j++)
                if (lane * PER + j < E) to[j] = out[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <class F>
static hipError_t by_members(int members, F f) {
    if (members <= 64) return f(std::integral_constant<int, 1>());
    if (members <= 128) return f(std::integral_constant<int, 2>());
    if (members <= 256) return f(std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 8>());
}

// Two workgroups of a compute unit's 32 wavefronts.
template <int PER>
static unsigned route_blocks(int64_t n) { return (unsigned)std::min<int64_t>((n + ROUTE_WAVES<PER> - 1) / ROUTE_WAVES<PER>, 8192 / ROUTE_WAVES<PER>); }

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        return by_members(a.members, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            const dim3 grid(route_blocks<PER>(a.n)), group(64 * ROUTE_WAVES<PER>);
            if (!a.bias && a.groups == 1) hipLaunchKernelGGL((route_kernel<decltype(t), PER, true>), grid, group, 0, s, a);
            else hipLaunchKernelGGL((route_kernel<decltype(t), PER, false>), grid, group, 0, s, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        return by_members(a.members, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            hipLaunchKernelGGL((route_backward_kernel<decltype(t), PER>), dim3(route_blocks<PER>(a.n)), dim3(64 * ROUTE_WAVES<PER>), 0, s, a);
            return hipGetLastError();
        });
    });
}

}  // namespace ens
