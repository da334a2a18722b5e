// Routing: a gate's scores choose members for each row, and weigh them.
//   s = softmax(x) or sigmoid(x) over the members; a member ranks by c = s + bias, or by x where there is no bias (s rises with x)
//   groups of neighbouring members rank by the sum of their one or two best c; members of the best groups stay
//   the k best c are chosen, the lowest member on equal ones; weight = scale s, or scale s / (sum of the chosen s)
// x of minus infinity or NaN: not a member of this row.
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

enum { SCORE_SOFTMAX = 0, SCORE_SIGMOID = 1 };
constexpr int ROUTE_WAVES = 4;

template <class R>
__device__ __forceinline__ R wave_max_of(R v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const R w = __shfl_xor(v, o, 64);
        v = w > v ? w : v;
    }
    return v;
}
template <class R>
__device__ __forceinline__ R wave_sum_of(R v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float exp_r(float v) { return expf(v); }
__device__ __forceinline__ double exp_r(double v) { return exp(v); }
__device__ __forceinline__ float log1p_r(float v) { return log1pf(v); }
__device__ __forceinline__ double log1p_r(double v) { return log1p(v); }

// A gate's value; not a member: minus infinity.
template <class R>
__device__ __forceinline__ R gate_value(float x) { return x > NONE ? (R)fminf(x, -LOWEST) : -(R)__builtin_inf(); }
template <class R>
__device__ __forceinline__ R sigmoid_of(R x) { return x >= 0 ? 1 / (1 + exp_r(-x)) : exp_r(x) / (1 + exp_r(x)); }
// Logarithm of the score up to a constant of the row.
template <class R>
__device__ __forceinline__ R log_score(int score, R x) {
    if (score == SCORE_SOFTMAX) return x;
    return x >= 0 ? -log1p_r(exp_r(-x)) : x - log1p_r(exp_r(x));
}

// The members of a row, member lane + 64 j in x[j] and its score in s[j].
template <class R, int PER>
__device__ __forceinline__ void row_scores(int score, const R (&x)[PER], R (&s)[PER]) {
    const R none = -(R)__builtin_inf();
    if (score == SCORE_SIGMOID) {
#pragma unroll
        for (int j = 0; j < PER; j++) s[j] = x[j] > none ? sigmoid_of(x[j]) : 0;
        return;
    }
    R m = none, sum = 0;
#pragma unroll
    for (int j = 0; j < PER; j++) m = x[j] > m ? x[j] : m;
    m = wave_max_of(m);
#pragma unroll
    for (int j = 0; j < PER; j++) {
        s[j] = x[j] > none ? exp_r(x[j] - m) : 0;
        sum += s[j];
    }
    sum = wave_sum_of(sum);
#pragma unroll
    for (int j = 0; j < PER; j++) s[j] = sum > 0 ? s[j] / sum : 0;
}

template <class T, int PER>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_kernel(const RouteArgs a) {
    typedef double R;
    __shared__ int counts[ROUTE_MAX_MEMBERS];
    __shared__ R ranks[ROUTE_WAVES][PER * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E = a.members;
    const R none = -(R)__builtin_inf();
    if (a.load) {
        for (int e = threadIdx.x; e < E; e += 64 * ROUTE_WAVES) counts[e] = 0;
        __syncthreads();
    }
    for (int64_t row = (int64_t)blockIdx.x * ROUTE_WAVES + wave; row < a.n; row += (int64_t)gridDim.x * ROUTE_WAVES) {
        const T* const gates = (const T*)a.gates + row * a.ld;
        R x[PER], s[PER], c[PER];
#pragma unroll
        for (int j = 0; j < PER; j++) x[j] = lane + 64 * j < E ? gate_value<R>(up(gates[lane + 64 * j])) : none;
        row_scores<R, PER>(a.score, x, s);
#pragma unroll
        for (int j = 0; j < PER; j++) {
            c[j] = none;
            if (x[j] > none) {
                c[j] = a.bias ? s[j] + (R)a.bias[lane + 64 * j] : a.groups > 1 ? s[j] : x[j];
                if (!(c[j] > none)) c[j] = none;
            }
        }
        if (a.groups > 1) {
            const int size = E / a.groups;
#pragma unroll
            for (int j = 0; j < PER; j++) ranks[wave][lane + 64 * j] = c[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            R first = none, second = none;
            if (lane < a.groups)
                for (int i = 0; i < size; i++) {
                    const R v = ranks[wave][lane * size + i];
                    if (v > first) { second = first; first = v; }
                    else if (v > second) second = v;
                }
            const R group = a.group_best == 2 && second > none ? first + second : first;
            int better = 0;
            for (int g = 0; g < a.groups; g++) {
                const R other = __shfl(group, g, 64);
                better += other > group || (other == group && g < lane);
            }
            const unsigned long long kept = __ballot(lane < a.groups && better < a.groups_kept);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < PER; j++) {
                const int e = lane + 64 * j;
                if (e < E && !(kept >> (e / size) & 1)) c[j] = none;
            }
        }
        int mine = -1;                                           // lane j keeps the j-th choice
        for (int i = 0; i < a.k; i++) {
            R best = none;
            int at = 0x7FFFFFFF;
#pragma unroll
            for (int j = 0; j < PER; j++)
                if (c[j] > best) { best = c[j]; at = lane + 64 * j; }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const R b = __shfl_xor(best, o, 64);
                const int t = __shfl_xor(at, o, 64);
                if (b > best || (b == best && t < at)) { best = b; at = t; }
            }
            if (!(best > none)) break;
            if (lane == i) mine = at;
#pragma unroll
            for (int j = 0; j < PER; j++)
                if (lane + 64 * j == at) c[j] = none;
        }
        R weight = 0;
        const R own = mine >= 0 ? gate_value<R>(up(gates[mine])) : none;
        if (a.renormalise) {
            const R l = mine >= 0 ? log_score(a.score, own) : none, top = wave_max_of(l);
            const R e = mine >= 0 ? exp_r(l - top) : 0, sum = wave_sum_of(e);
            weight = mine >= 0 ? e / sum : 0;
        } else {
#pragma unroll
            for (int j = 0; j < PER; j++) {
                const R v = __shfl(s[j], mine & 63, 64);
                if (mine >= 0 && mine >> 6 == j) weight = v;
            }
        }
        if (lane < a.k) {
            a.chosen[row * a.k + lane] = mine;
            a.weights[row * a.k + lane] = (float)(weight * (R)a.scale);
            if (a.load && mine >= 0) atomicAdd(&counts[mine], 1);
        }
    }
    if (a.load) {
        __syncthreads();
        for (int e = threadIdx.x; e < E; e += 64 * ROUTE_WAVES)
            if (counts[e]) atomicAdd(&a.load[e], counts[e]);
    }
}

// u_j = scale dL/dw_j.  Renormalised: r = softmax over the chosen of ln s, dL/d(ln s_j) = r_j (u_j - sum r u); softmax: that is dL/dx_j,
// sigmoid: times 1 - s_j.  As they are: softmax dL/dx_e = s_e (u_e - sum u_j s_j), sigmoid dL/dx_j = u_j s_j (1 - s_j).
// The choice itself has no derivative.
template <class T, int PER>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_backward_kernel(const RouteArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E = a.members;
    for (int64_t row = (int64_t)blockIdx.x * ROUTE_WAVES + wave; row < a.n; row += (int64_t)gridDim.x * ROUTE_WAVES) {
        const T* const gates = (const T*)a.gates + row * a.ld;
        T* const out = (T*)a.d_gates + row * a.ld_d;
        int mine = lane < a.k ? a.chosen[row * a.k + lane] : -1;
        if (mine < 0 || mine >= E) mine = -1;
        const float u = mine >= 0 ? a.scale * a.d_weights[row * a.k + lane] : 0.f;
        const float own = mine >= 0 ? gate_value<float>(up(gates[mine])) : NONE;
        if (!(own > NONE)) mine = -1;
        float d[PER], slot = 0.f;                                // of the members; of this lane's choice
#pragma unroll
        for (int j = 0; j < PER; j++) d[j] = 0.f;
        if (a.renormalise) {
            const float l = mine >= 0 ? log_score(a.score, own) : NONE, top = wave_max_of(l);
            const float e = mine >= 0 ? exp_r(l - top) : 0.f, sum = wave_sum_of(e);
            const float r = mine >= 0 ? e / sum : 0.f;
            const float mean = wave_sum_of(r * u);
            slot = r * (u - mean);
            if (a.score == SCORE_SIGMOID && mine >= 0) slot *= sigmoid_of(-own);
        } else if (a.score == SCORE_SIGMOID) {
            if (mine >= 0) slot = u * sigmoid_of(own) * sigmoid_of(-own);
        } else {
            float x[PER], s[PER], part = 0.f;
#pragma unroll
            for (int j = 0; j < PER; j++) x[j] = lane + 64 * j < E ? gate_value<float>(up(gates[lane + 64 * j])) : NONE;
            row_scores<float, PER>(a.score, x, s);
#pragma unroll
            for (int j = 0; j < PER; j++) {
                const float v = __shfl(s[j], mine & 63, 64);
                if (mine >= 0 && mine >> 6 == j) part = v;
            }
            slot = u * part;
            const float mean = wave_sum_of(slot);
#pragma unroll
            for (int j = 0; j < PER; j++) d[j] = -s[j] * mean;
        }
        for (int i = 0; i < a.k; i++) {                          // a member that was chosen twice gets both
            const int e = __builtin_amdgcn_readlane(mine, i);
            const float v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(slot), i));
            if (e < 0) continue;
#pragma unroll
            for (int j = 0; j < PER; j++)
                if (lane + 64 * j == e) d[j] += v;
        }
#pragma unroll
        for (int j = 0; j < PER; j++)
            if (lane + 64 * j < E) out[lane + 64 * j] = (T)d[j];
    }
}

template <class F>
static hipError_t by_members(int members, F f) {
    if (members <= 64) return f(std::integral_constant<int, 1>());
    if (members <= 128) return f(std::integral_constant<int, 2>());
    if (members <= 256) return f(std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 8>());
}

static unsigned route_blocks(int64_t n) { return (unsigned)std::min<int64_t>((n + ROUTE_WAVES - 1) / ROUTE_WAVES, 2048); }

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        return by_members(a.members, [&](auto per) {
            hipLaunchKernelGGL((route_kernel<decltype(t), decltype(per)::value>), dim3(route_blocks(a.n)), dim3(64 * ROUTE_WAVES), 0, s, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        return by_members(a.members, [&](auto per) {
            hipLaunchKernelGGL((route_backward_kernel<decltype(t), decltype(per)::value>), dim3(route_blocks(a.n)), dim3(64 * ROUTE_WAVES), 0, s, a);
            return hipGetLastError();
        });
    });
}

}  // namespace ens
