// Distillation: a student's logits x against the classes that a teacher kept of a row, with the logarithms t of their probabilities.
//   p = softmax(x / T);  q = softmax(t) over the kept classes (tail off), or q = e^t and q_0 = 1 - sum q (0 below 2^-21) for all the others (tail on)
//   loss = T^2 (sum q ln(q / p) [+ q_0 ln(q_0 / p_0)]),  p_0 = sum of p over the classes that were not kept
//   dloss/dx_c = T (S p_c - q_c), S = sum q (+ q_0);  with tail, for a class that was not kept, T (S - q_0 / p_0) p_c
// A class that is listed twice has the sum of its q.  An entry outside the row is not there.  With tail on and no other class, or all others at minus
// infinity, the tail counts nothing.  A row without a kept class of any probability (tail off), or without a finite logit, counts nothing.
//
// With tail the kept classes and the others each have a maximum and a sum of their own, E = sum e^((x - max_E) / T) and R = sum e^((x - max_R) / T): what a sure
// student leaves to the others is far below what fp32 holds beside the row's maximum, but its logarithm is not, and neither are the shares of the others in it.
// With odds = ln (E e^(max_E / T)) - ln (R e^(max_R / T)), p of all kept classes 1 / (1 + e^-odds) and p_0 = 1 / (1 + e^odds), nothing is divided by what can vanish:
//   dloss/dx_c = T (sum q p_0 - q_0 (1 - p_0)) e^((x_c - max_R) / T) / R   for a class that was not kept
//   ln p_c = (x_c - max_E) / T - ln E + ln (1 - p_0)                       for one that was
//
// Bound by memory: a row read, and its gradient written.  A workgroup keeps a row in registers from its maximum through the sums to the gradient, so that
// it is read once (up to 131 072 classes of 16 bits, half as many of fp32), with as many threads as leave the most rows to a compute unit at a time;
// longer rows, and few of the longest, go in parts of 2 048 pieces of 16 bytes, which are read twice.  The teacher's record is read by the first
// wavefront while the others' loads are on their way.
// Gradient with the loss, k = 50, as calls: 4 096 rows of 128 000 bf16 classes 423 us (4.96 TB/s of what has to move; torch's copy of them 400), with the tail
// 447; 1 021 rows of 50 001 47 and 48 us (4.3 TB/s, two rows a compute unit at a time, whose ends leave it idle); in parts, read twice, 700 rows of 200 000 154 and
// 158, 2 048 rows of 151 936 344 and 349 (3.6 TB/s).  Backward by itself 42, 102 and 225 us for the last three (4.8 to 5.5 TB/s).
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

constexpr int KEPT_LANES = DISTILL_MAX_K / 64;
constexpr int CUS = 256;                                         // compute units

// What less than this is left of 1 is not told from the roundings of q and of their sum; the distance of classes at the lowest value, as a mask leaves them, would
// make it a loss of 1e30.
constexpr float LEAST_REST = 0x1p-21f;

// The teacher's record of a row in LDS, as a wavefront leaves it: class (or -1) and q of k entries, the sum of q, q_0, and the sum of q ln q.
struct Record {
    int* index;
    float* q;
    float* sums;
};
// mark(c) marks class c and says whether it was marked; nullptr for kernels without marks.
template <class F>
__device__ __forceinline__ void read_record(const DistillArgs& a, int64_t row, int lane, const Record& r, F mark) {
    constexpr bool MARKS = !std::is_same<F, std::nullptr_t>::value;
    const int32_t* const index = a.index + row * a.k;
    const float* const log_probs = a.log_probs + row * a.k;
    int c[KEPT_LANES];
    float q[KEPT_LANES], top = NONE, sum = 0.f;
#pragma unroll
    for (int i = 0; i < KEPT_LANES; i++) {
        const int j = 64 * i + lane;
        c[i] = j < a.k ? index[j] : -1;
        q[i] = j < a.k ? log_probs[j] : NONE;
        if (c[i] < 0 || c[i] >= a.classes) {
            c[i] = -1;
            q[i] = NONE;
        }
        top = fmaxf(top, q[i]);
    }
    top = a.tail ? 0.f : lanes_max(top);
#pragma unroll
    for (int i = 0; i < KEPT_LANES; i++) {
        q[i] = q[i] == NONE ? 0.f : expf(q[i] - top);
        sum += q[i];
    }
    if (!a.tail) {
        sum = lanes_sum(sum);
        const float scale = sum == 0.f ? 1.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < KEPT_LANES; i++) q[i] *= scale;
    }
    // does a class come twice?
    bool twice = false;
    if constexpr (MARKS) {
        bool again = false;
#pragma unroll
        for (int i = 0; i < KEPT_LANES; i++)
            if (c[i] >= 0) again = mark(c[i]) || again;
        twice = __ballot(again) != 0;
    } else {
        int times[KEPT_LANES] = {};                              // that an entry's class comes
        auto count = [&](auto groups) {
            constexpr int GROUPS = decltype(groups)::value;
#pragma unroll
            for (int o = 0; o < GROUPS; o++) {
                const int entries = min(64, a.k - 64 * o);
                for (int l = 0; l < entries; l++) {
                    const int other = __builtin_amdgcn_readlane(c[o], l);
#pragma unroll
                    for (int i = 0; i < GROUPS; i++) times[i] += c[i] == other;
                }
            }
        };
        if (a.k <= 64) count(std::integral_constant<int, 1>());
        else count(std::integral_constant<int, KEPT_LANES>());
        bool again = false;
#pragma unroll
        for (int i = 0; i < KEPT_LANES; i++) again = again || (c[i] >= 0 && times[i] > 1);
        twice = __ballot(again) != 0;
    }
    float mass = 0.f, entropy = 0.f;
#pragma unroll
    for (int i = 0; i < KEPT_LANES; i++) {
        if (64 * i >= a.k) break;
        const int j = 64 * i + lane;
        float all = q[i];
        bool first = c[i] >= 0;
        if (twice) {                                             // the first entry of a class takes what the later ones have
            all = 0.f;
#pragma unroll
            for (int o = 0; o < KEPT_LANES; o++) {
                const int entries = min(64, a.k - 64 * o);
                for (int l = 0; l < entries; l++) {
                    const bool same = c[i] == __builtin_amdgcn_readlane(c[o], l);
                    all += same ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(q[o]), l)) : 0.f;
                    if (64 * o + l < j) first = first && !same;
                }
            }
        }
        if (!first) all = 0.f;
        if (j < a.k) {
            r.index[j] = first ? c[i] : -1;
            r.q[j] = all;
        }
        mass += all;
        if (all != 0.f) entropy += all * logf(all);
    }
    mass = lanes_sum(mass);
    entropy = lanes_sum(entropy);
    if (lane == 0) {
        r.sums[0] = mass;
        r.sums[1] = a.tail && 1.f - mass >= LEAST_REST ? 1.f - mass : 0.f;
        r.sums[2] = entropy;
    }
}

// A bit for each class, set for those that are kept: bit HEADS + c - head, so that a piece's bits stand together, in a byte or half a byte.
// Piece `first` + tid, `first` even.
template <class T, int THREADS>
__device__ __forceinline__ uint32_t piece_marks(const uint32_t* marks, int first, int tid) {
    const uint8_t* const bytes = (const uint8_t*)marks;
    constexpr int HEADS = Row<T, THREADS>::HEADS;
    if constexpr (PIECE<T> == 8) return bytes[HEADS / 8 + tid + first];
    else return bytes[((HEADS / 4 + tid) >> 1) + (first >> 1)] >> (4 * ((HEADS / 4 + tid) & 1)) & 15u;
}
template <class T, int THREADS>
static __host__ __device__ int mark_words(int pieces) { return ((pieces + 1) * PIECE<T> + Row<T, THREADS>::HEADS + 31) / 32; }

// What a row's record and the student's logits of its classes come to: sum of q, q_0, sum of q ln q; max_E and E (with tail).
struct Kept { float mass, rest, entropy, max, sum; };
__device__ __forceinline__ Kept kept_of(const Record& r, float max, float sum) { return Kept{r.sums[0], r.sums[1], r.sums[2], max, sum}; }
// ln of what the kept classes have over what the others have; plus infinity where the others have nothing, minus infinity where the kept ones (or both) have.
__device__ __forceinline__ float log_odds(const Kept& kept, float mx, float sum, float temperature) {
    if (kept.sum == 0.f) return NONE;
    if (sum == 0.f) return -NONE;
    return 2.f * ((0.5f * kept.max - 0.5f * mx) / temperature) + (logf(kept.sum) - logf(sum));     // (halves as in row_loss)
}
// A row's loss.  mx, sum: max_R and R with tail, otherwise of all classes.  cross: sum of q (x / 2 - max / 2) over the kept classes, max max_E with
// tail, otherwise mx.  Distances are halved, since those of two fp32 values may not be one, and divided by nothing, since they are multiplied by T in the end.
template <bool TAIL>
__device__ __forceinline__ float row_loss(const Kept& kept, float cross, float mx, float sum, float odds, float T) {
    float shared = kept.entropy, far = -cross;                   // what is multiplied by T^2, and by 2 T
    if constexpr (TAIL) {
        const float mass = kept.mass, rest = sum == 0.f ? 0.f : kept.rest;
        if (kept.sum == 0.f && sum == 0.f) return 0.f;
        if (rest > 0.f) shared += rest * logf(rest);
        if (kept.sum == 0.f) return mass != 0.f ? mass * -NONE : T * T * shared;     // p_0 = 1
        // -ln p_0 = odds + ln (1 + e^-odds), -ln (1 - p_0) = ln (1 + e^-odds), with both signs the other way round where odds are below 0
        shared += mass * logf(kept.sum) + (mass + rest) * log1pf(expf(-fabsf(odds)));
        if (sum != 0.f) {
            const float tilt = odds < 0.f ? -mass : rest;
            shared += tilt * (logf(kept.sum) - logf(sum));
            far += tilt * (0.5f * kept.max - 0.5f * mx);
        }
    } else {
        if (sum == 0.f || kept.mass == 0.f) return 0.f;
        shared += kept.mass * logf(sum);
    }
    return T * T * shared + 2.f * T * far;
}
// What multiplies e^((x - max) / T) in the gradient of a class that was not kept, and of one that was, whose maximum is max_E if they stand `apart`.
struct Factors { float other, kept; };
template <bool TAIL>
__device__ __forceinline__ Factors factors(const Kept& kept, float sum, float odds, float weight, bool apart = TAIL) {
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    if constexpr (!TAIL) return Factors{weight * kept.mass * inverse, weight * kept.mass * inverse};
    const float less = expf(-fabsf(odds)), large = 1.f / (1.f + less), small = less * large;
    const float in = odds < 0.f ? small : large, out = odds < 0.f ? large : small;     // 1 - p_0, p_0
    const float rest = sum == 0.f ? 0.f : kept.rest;
    const float share = !apart ? out * inverse : kept.sum == 0.f ? 0.f : in / kept.sum;
    return Factors{weight * (kept.mass * out - rest * in) * inverse, weight * (kept.mass + rest) * share};
}
// Odds up to which the backward pass takes p of the kept classes from the others' maximum and sum, as p_0 e^((x - max_R) / T) / R, which takes no other logits: the
// odds of the state are rounded at their size, to 2^-21 here, and such a p is off by as much of itself.
constexpr float NEAR_ODDS = 16.f;

// LDS of a workgroup: two floats for each of 16 wavefronts, the record, the marks
static __host__ __device__ int record_words(int k) { return 32 + 2 * k + 3; }
__device__ __forceinline__ Record record_in(int* lds, int k) { return Record{lds + 32, (float*)lds + 32 + k, (float*)lds + 32 + 2 * k}; }
// Two reductions between the same barriers.
template <int THREADS>
__device__ __forceinline__ void group_max(float& v, float& w, float* box) {
    v = lanes_max(v);
    w = lanes_max(w);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            box[threadIdx.x >> 6] = v;
            box[16 + (threadIdx.x >> 6)] = w;
        }
        __syncthreads();
        v = box[0];
        w = box[16];
#pragma unroll
        for (int i = 1; i < THREADS / 64; i++) {
            v = fmaxf(v, box[i]);
            w = fmaxf(w, box[16 + i]);
        }
    }
}
template <int THREADS>
__device__ __forceinline__ void group_sum(float& v, float& w, float* box) {
    v = lanes_sum(v);
    w = lanes_sum(w);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            box[threadIdx.x >> 6] = v;
            box[16 + (threadIdx.x >> 6)] = w;
        }
        __syncthreads();
        v = box[0];
        w = box[16];
#pragma unroll
        for (int i = 1; i < THREADS / 64; i++) {
            v += box[i];
            w += box[16 + i];
        }
    }
}

// A workgroup a row, the row in registers between its maximum, its sums and its gradient.  The registers that a thread may use are stated by the
// wavefronts that are to fit: with 169 instead of 126 a compute unit had one row of 50 001 classes at a time instead of two, 108 us instead of 68.
template <class T, bool TAIL, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS, PIECES == 28 ? 3 : PIECES == 16 ? 4 : PIECES == 8 ? 5 : 6) void distill_held_kernel(const DistillArgs a) {
    extern __shared__ int lds[];
    const int tid = threadIdx.x, k = a.k;
    constexpr int KEPT = (DISTILL_MAX_K + THREADS - 1) / THREADS;
    float* const box = (float*)lds;
    const Record record = record_in(lds, k);
    uint32_t* const marks = (uint32_t*)lds + record_words(k);
    const float cooling = 1.f / a.temperature;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.logits + row * a.ld;
        const Row<T, THREADS> x(p, a.classes);
        Held<T, THREADS, PIECES> held;
        held.load(x, tid);
        const int shift = x.HEADS - x.head;
        if constexpr (TAIL) {
            if (tid < 64) {
                for (int i = tid; i < mark_words<T, THREADS>(THREADS * PIECES); i += 64) marks[i] = 0;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                read_record(a, row, tid, record, [&](int c) {
                    const uint32_t bit = 1u << ((c + shift) & 31);
                    return (atomicOr(&marks[(c + shift) >> 5], bit) & bit) != 0;
                });
            }
        } else if (tid < 64) read_record(a, row, tid, record, nullptr);
        group_sync<THREADS>();
        float at_kept[KEPT], mx, most = LOWEST;
#pragma unroll
        for (int i = 0; i < KEPT; i++) {
            const int j = tid + i * THREADS, at = j < k ? record.index[j] : -1;
            at_kept[i] = at >= 0 ? up(p[at]) : NONE;
        }
        if constexpr (TAIL) {
            held.hide(x, held.at >= 0 && (marks[(held.at + shift) >> 5] >> ((held.at + shift) & 31) & 1),
                      [&](int piece) { return piece_marks<T, THREADS>(marks, piece, tid); });
            mx = held.max(x);
#pragma unroll
            for (int i = 0; i < KEPT; i++) most = fmaxf(most, at_kept[i]);
            group_max<THREADS>(mx, most, box);
        } else mx = group_max<THREADS>(held.max(x), box);
        const Exp power(mx, cooling), power_kept(TAIL ? most : mx, cooling);
        float sum = power(held.one), sum_kept = 0.f;
        held.each(x, [&](float (&v)[PIECE<T>], int) {
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) v[e] = power(v[e]);
            sum += sum_of(v);
        });
        if constexpr (TAIL) {
#pragma unroll
            for (int i = 0; i < KEPT; i++) sum_kept += power_kept(at_kept[i]);
            group_sum<THREADS>(sum, sum_kept, box);
        } else sum = group_sum<THREADS>(sum, box);
        sum *= power.off();
        const Kept kept = kept_of(record, most, sum_kept * power_kept.off());
        const float odds = TAIL ? log_odds(kept, mx, sum, a.temperature) : 0.f;
        float cross = 0.f;
#pragma unroll
        for (int i = 0; i < KEPT; i++) {
            const int j = tid + i * THREADS;
            if (j < k && record.q[j] != 0.f) cross += record.q[j] * (0.5f * at_kept[i] - 0.5f * power_kept.m);
        }
        cross = group_sum<THREADS>(cross, box);
        if (tid == 0) {
            a.loss[row] = row_loss<TAIL>(kept, cross, mx, sum, odds, a.temperature);
            a.state[row * 3] = mx;
            a.state[row * 3 + 1] = logf(sum);
            a.state[row * 3 + 2] = odds;
        }
        if (a.d_logits) {
            T* const out = (T*)a.d_logits + row * a.ld_d;
            const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature;
            const bool none = weight == 0.f || (sum == 0.f && (!TAIL || odds == NONE));
            const Factors f = factors<TAIL>(kept, sum, odds, weight);
            const float other = none ? 0.f : f.other * power.off(), own = f.kept * power_kept.off();
            if (none) held.clear();
            held.map(x, tid, out, [&](float v) { return other * power(v); });
            group_sync<THREADS>();
            if (!none)
#pragma unroll
                for (int i = 0; i < KEPT; i++) {
                    const int j = tid + i * THREADS;
                    if (j < k && record.index[j] >= 0) out[record.index[j]] = (T)(own * power_kept(at_kept[i]) - weight * record.q[j]);
                }
        }
        group_sync<THREADS>();
    }
}

// The rows in parts, for rows that are too long for a workgroup's registers or too few: first every part's maximum and sum and the logits of the
// kept classes go to the workspace, then every part's workgroup joins them and writes its part of the gradient, the first one the loss.  The second
// step by itself, from the state, is the backward pass; where that writes over the logits of several parts, the kept classes wait for a launch of their own, since
// with tail every one of them needs the logits of all.  A part is in registers too.
constexpr int PART_THREADS = 256, PART_PIECES = 8;
struct Parts {
    int parts, length;                                           // of every part but the last
    bool kept_later;
    __host__ __device__ int64_t row_floats(int k) const { return (int64_t)parts * 4 + k; }     // maximum and sum of all (with tail of the others), of the kept; the kept classes' logits
};

template <class T, bool TAIL>
__global__ __launch_bounds__(PART_THREADS, 6) void distill_part_kernel(const DistillArgs a, const Parts split) {
    extern __shared__ int lds[];
    const int tid = threadIdx.x, k = a.k;
    float* const box = (float*)lds;
    uint32_t* const marks = (uint32_t*)lds + 32;
    const float cooling = 1.f / a.temperature;
    for (int64_t job = blockIdx.x; job < a.n * split.parts; job += gridDim.x) {
        const int64_t row = job / split.parts;
        const int part = (int)(job - row * split.parts), first = part * split.length, length = min(split.length, a.classes - first);
        const T* const p = (const T*)a.logits + row * a.ld + first;
        const Row<T, PART_THREADS> x(p, length);
        Held<T, PART_THREADS, PART_PIECES> held;
        held.load(x, tid);
        float* const out = (float*)a.workspace + row * split.row_floats(k);
        const int shift = x.HEADS - x.head;
        if (TAIL) {
            for (int i = tid; i < mark_words<T, PART_THREADS>(PART_THREADS * PART_PIECES); i += PART_THREADS) marks[i] = 0;
            __syncthreads();
        }
        float at_kept = NONE, most = LOWEST, mx;                 // (PART_THREADS entries at most)
        if (tid < k) {
            const int64_t at = (int64_t)a.index[row * k + tid] - first;
            if (at >= 0 && at < length) {
                const float v = up(p[at]);
                out[split.parts * 4 + tid] = v;
                const uint32_t bit = 1u << ((at + shift) & 31);
                if (TAIL && !(atomicOr(&marks[(at + shift) >> 5], bit) & bit)) at_kept = v;     // a class that comes twice counts once
            }
        }
        if constexpr (TAIL) {
            __syncthreads();
            held.hide(x, held.at >= 0 && (marks[(held.at + shift) >> 5] >> ((held.at + shift) & 31) & 1),
                      [&](int piece) { return piece_marks<T, PART_THREADS>(marks, piece, tid); });
            mx = held.max(x);
            most = fmaxf(most, at_kept);
            group_max<PART_THREADS>(mx, most, box);
        } else mx = group_max<PART_THREADS>(held.max(x), box);
        const Exp power(mx, cooling), power_kept(most, cooling);
        float sum = power(held.one), sum_kept = TAIL ? power_kept(at_kept) : 0.f;
        held.each(x, [&](float (&v)[PIECE<T>], int) {
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) v[e] = power(v[e]);
            sum += sum_of(v);
        });
        if constexpr (TAIL) group_sum<PART_THREADS>(sum, sum_kept, box);
        else sum = group_sum<PART_THREADS>(sum, box);
        if (tid == 0) {
            out[part * 4] = mx;
            out[part * 4 + 1] = sum * power.off();
            out[part * 4 + 2] = most;
            out[part * 4 + 3] = sum_kept * power_kept.off();
        }
        __syncthreads();
    }
}
static_assert(DISTILL_MAX_K <= PART_THREADS, "a thread an entry");

template <class T, bool TAIL, bool JOIN, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS, 6) void distill_gradient_kernel(const DistillArgs a, const Parts split) {
    extern __shared__ int lds[];
    __shared__ float found[4];
    constexpr int KEPT = (DISTILL_MAX_K + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, k = a.k;
    float* const box = (float*)lds;
    const Record record = record_in(lds, k);
    const float cooling = 1.f / a.temperature;
    const int per_row = a.d_logits ? split.parts : 1;            // the first part alone has the loss
    for (int64_t job = blockIdx.x; job < a.n * per_row; job += gridDim.x) {
        const int64_t row = job / per_row;
        const int part = (int)(job - row * per_row), first = part * split.length, length = min(split.length, a.classes - first);
        const float* const from = (const float*)a.workspace + row * split.row_floats(k);
        const T* const p = (const T*)a.logits + row * a.ld + first;
        const Row<T, THREADS> x(p, length);
        Held<T, THREADS, PIECES> held;
        const bool gradient = !JOIN || a.d_logits;
        if (gradient) held.load(x, tid);
        if (tid < 64) {
            read_record(a, row, lane, record, nullptr);
            if (JOIN) {
                constexpr int SETS = TAIL ? 2 : 1;
                float v[4];                                      // as `found` and a part's four floats
#pragma unroll
                for (int e = 0; e < 2 * SETS; e++) v[e] = e % 2 ? 0.f : LOWEST;
                for (int i = lane; i < split.parts; i += 64)
#pragma unroll
                    for (int e = 0; e < 2 * SETS; e += 2) v[e] = fmaxf(v[e], from[i * 4 + e]);
#pragma unroll
                for (int e = 0; e < 2 * SETS; e += 2) v[e] = lanes_max(v[e]);
                for (int i = lane; i < split.parts; i += 64)
#pragma unroll
                    for (int e = 0; e < 2 * SETS; e += 2)
                        v[e + 1] += from[i * 4 + e + 1] * Exp(v[e], cooling).less(from[i * 4 + e]);
#pragma unroll
                for (int e = 0; e < 2 * SETS; e += 2) {
                    v[e + 1] = lanes_sum(v[e + 1]);
                    if (lane == 0) {
                        found[e] = v[e];
                        found[e + 1] = v[e + 1];
                    }
                }
                if (part == 0) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    const float most = TAIL ? v[2] : v[0];
                    float cross = 0.f;
                    for (int j = lane; j < k; j += 64)
                        if (record.q[j] != 0.f) cross += record.q[j] * (0.5f * from[split.parts * 4 + j] - 0.5f * most);
                    cross = lanes_sum(cross);
                    if (lane == 0) {
                        const Kept kept = kept_of(record, most, TAIL ? v[3] : 0.f);
                        const float odds = TAIL ? log_odds(kept, v[0], v[1], a.temperature) : 0.f;
                        a.loss[row] = row_loss<TAIL>(kept, cross, v[0], v[1], odds, a.temperature);
                        a.state[row * 3] = v[0];
                        a.state[row * 3 + 1] = logf(v[1]);
                        a.state[row * 3 + 2] = odds;
                    }
                }
            }
        }
        group_sync<THREADS>();
        if (gradient) {
            T* const out = (T*)a.d_logits + row * a.ld_d + first;
            const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature;
            const float mx = JOIN ? found[0] : a.state[row * 3], sum = JOIN ? found[1] : expf(a.state[row * 3 + 1]);
            float odds = TAIL && !JOIN ? a.state[row * 3 + 2] : 0.f;
            // other parts' logits are of use for E, as far as they are not gradients by now
            const bool far = TAIL && !JOIN && !(fabsf(odds) <= NEAR_ODDS), later = far && split.kept_later, all = far && !later;
            float at_kept[KEPT], most = LOWEST, sum_kept = 0.f;
            int at[KEPT];
#pragma unroll
            for (int i = 0; i < KEPT; i++) {
                const int j = tid + i * THREADS, c = j < k ? record.index[j] : -1;
                const int here = c - first;
                at[i] = c >= 0 && here >= 0 && here < length ? here : -1;
                at_kept[i] = !(all ? c >= 0 : at[i] >= 0) ? NONE : JOIN ? from[split.parts * 4 + j] : up(p[here]);
                most = fmaxf(most, at_kept[i]);
            }
            if (JOIN && TAIL) {
                most = found[2];
                sum_kept = found[3];
            } else if (all) {
                most = group_max<THREADS>(most, box);
                const Exp power(most, cooling);
#pragma unroll
                for (int i = 0; i < KEPT; i++) sum_kept += power(at_kept[i]);
                sum_kept = group_sum<THREADS>(sum_kept, box) * power.off();
            }
            const Kept kept = kept_of(record, most, sum_kept);
            if (TAIL && JOIN) odds = log_odds(kept, mx, sum, a.temperature);
            const bool none = weight == 0.f || (sum == 0.f && (!TAIL || odds == NONE));
            const bool apart = TAIL && (JOIN || far);            // the kept classes by max_E and E
            const Factors f = factors<TAIL>(kept, sum, odds, weight, apart);
            group_sync<THREADS>();                               // out may be p
            const Exp power(mx, cooling), power_kept(apart ? most : mx, cooling);
            const float other = none ? 0.f : f.other * power.off(), own = f.kept * power_kept.off();
            if (none) held.clear();
            held.map(x, tid, out, [&](float v) { return other * power(v); });
            group_sync<THREADS>();
#pragma unroll
            for (int i = 0; i < KEPT; i++) {
                if (at[i] < 0) continue;
                if (later) out[at[i]] = (T)at_kept[i];           // as it was
                else if (!none) out[at[i]] = (T)(own * power_kept(at_kept[i]) - weight * record.q[tid + i * THREADS]);
            }
        }
        group_sync<THREADS>();
    }
}

// The kept classes of rows whose other gradients are written and whose odds are far, a wavefront a row.
template <class T>
__global__ __launch_bounds__(64) void distill_kept_kernel(const DistillArgs a) {
    extern __shared__ int lds[];
    constexpr int KEPT = DISTILL_MAX_K / 64;
    const Record record = record_in(lds, a.k);
    const int lane = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const float sum = expf(a.state[row * 3 + 1]), odds = a.state[row * 3 + 2];
        if (fabsf(odds) <= NEAR_ODDS) continue;
        const T* const p = (const T*)a.logits + row * a.ld;
        T* const out = (T*)a.d_logits + row * a.ld_d;
        read_record(a, row, lane, record, nullptr);
        group_sync<64>();
        float at_kept[KEPT], most = LOWEST, sum_kept = 0.f;
        int at[KEPT];
#pragma unroll
        for (int i = 0; i < KEPT; i++) {
            at[i] = lane + 64 * i < a.k ? record.index[lane + 64 * i] : -1;
            at_kept[i] = at[i] >= 0 ? up(p[at[i]]) : NONE;
            most = fmaxf(most, at_kept[i]);
        }
        const Exp power(lanes_max(most), 1.f / a.temperature);
#pragma unroll
        for (int i = 0; i < KEPT; i++) sum_kept += power(at_kept[i]);
        const Kept kept = kept_of(record, power.m, lanes_sum(sum_kept) * power.off());
        const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature;
        const bool none = weight == 0.f || (sum == 0.f && odds == NONE);
        const float own = factors<true>(kept, sum, odds, weight).kept * power.off();
#pragma unroll
        for (int i = 0; i < KEPT; i++)
            if (at[i] >= 0) out[at[i]] = none ? (T)0.f : (T)(own * power(at_kept[i]) - weight * record.q[lane + 64 * i]);
        group_sync<64>();
    }
}

// Parts as long as a workgroup holds, or some 1 024 of them, of 4 096 classes at least.
static Parts split_rows(int64_t n, int classes, int dtype) {
    const int64_t piece = dtype == 0 ? 4 : 8, most = (classes + 4095) / 4096, want = std::max<int64_t>(1, 1024 / n);
    const int parts = (int)std::max<int64_t>((classes / piece + PART_THREADS * PART_PIECES - 1) / (PART_THREADS * PART_PIECES), std::min(most, want));
    if (parts <= 1) return Parts{1, classes, false};
    int length = ((classes + parts - 1) / parts + 63) / 64 * 64;
    length = std::min<int>(length, PART_THREADS * PART_PIECES * piece);
    return Parts{(classes + length - 1) / length, length, false};
}

// A row a workgroup holds it: with 512 threads whatever the rows are, with 1 024 (where a compute unit has one such row at a time) from some rows on.
// As calls from Python, whole and in parts, loss and gradient: a row of 64 000 bf16 classes 15.7 and 18.9 us, 200 of them 20.7 and 23.3;
// a row of 128 000 20.7 and 19.0, 64 of them 23.8 and 19.0, 200 of them 28.6 and 34.9.
static bool held(int64_t n, int classes, int dtype) {
    const int pieces = classes / (dtype == 0 ? 4 : 8);
    return pieces <= 512 * 16 || (pieces <= 1024 * 16 && n >= 160);
}

int64_t distill_workspace(int64_t n, int classes, int k, int dtype) {
    return held(n, classes, dtype) ? 0 : n * split_rows(n, classes, dtype).row_floats(k) * (int64_t)sizeof(float);
}

template <class T, bool TAIL, int THREADS, int PIECES>
static hipError_t launch_held(const DistillArgs& a, hipStream_t s) {
    const int lds = 4 * (record_words(a.k) + (TAIL ? mark_words<T, THREADS>(THREADS * PIECES) : 0));
    hipLaunchKernelGGL((distill_held_kernel<T, TAIL, THREADS, PIECES>), dim3((unsigned)std::min<int64_t>(a.n, 8192)), dim3(THREADS), lds, s, a);
    return hipGetLastError();
}

template <class T, bool TAIL>
static hipError_t launch_distill_as(const DistillArgs& a, hipStream_t s) {
    if (held(a.n, a.classes, a.dtype)) {
        const int pieces = a.classes / PIECE<T>;
        if (pieces <= 64 * 4) return launch_held<T, TAIL, 64, 4>(a, s);
        if (pieces <= 256 * 4) return launch_held<T, TAIL, 256, 4>(a, s);
        if (pieces <= 256 * 8) return launch_held<T, TAIL, 256, 8>(a, s);
        if (pieces <= 256 * 16) return launch_held<T, TAIL, 256, 16>(a, s);
        if (pieces <= 256 * 28 && 3 * ((a.n + 3 * CUS - 1) / (3 * CUS)) <= 2 * ((a.n + 2 * CUS - 1) / (2 * CUS))) return launch_held<T, TAIL, 256, 28>(a, s);
        if (pieces <= 512 * 16) return launch_held<T, TAIL, 512, 16>(a, s);
        return launch_held<T, TAIL, 1024, 16>(a, s);
    }
    const Parts split = split_rows(a.n, a.classes, a.dtype);
    const dim3 grid((unsigned)std::min<int64_t>(a.n * split.parts, 1 << 16)), group(PART_THREADS);
    const int lds = 4 * (32 + (TAIL ? mark_words<T, PART_THREADS>(PART_THREADS * PART_PIECES) : 0));
    hipLaunchKernelGGL((distill_part_kernel<T, TAIL>), grid, group, lds, s, a, split);
    const dim3 joins((unsigned)std::min<int64_t>(a.n * (a.d_logits ? split.parts : 1), 1 << 16));
    hipLaunchKernelGGL((distill_gradient_kernel<T, TAIL, true, PART_THREADS, PART_PIECES>), joins, group, 4 * record_words(a.k), s, a, split);
    return hipGetLastError();
}
hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) { return a.tail ? launch_distill_as<decltype(t), true>(a, s) : launch_distill_as<decltype(t), false>(a, s); });
}

template <class T, bool TAIL>
static hipError_t launch_backward_as(const DistillArgs& a, hipStream_t s) {
    if (a.classes / PIECE<T> <= 64 * 4) {                        // a wavefront a row
        const dim3 rows((unsigned)std::min<int64_t>(a.n, 1 << 16));
        hipLaunchKernelGGL((distill_gradient_kernel<T, TAIL, false, 64, 4>), rows, dim3(64), 4 * record_words(a.k), s, a, Parts{1, a.classes, false});
        return hipGetLastError();
    }
    Parts split = split_rows(a.n, a.classes, a.dtype);
    split.kept_later = TAIL && split.parts > 1 && a.d_logits == a.logits;
    const dim3 grid((unsigned)std::min<int64_t>(a.n * split.parts, 1 << 16));
    hipLaunchKernelGGL((distill_gradient_kernel<T, TAIL, false, PART_THREADS, PART_PIECES>), grid, dim3(PART_THREADS), 4 * record_words(a.k), s, a, split);
    if (split.kept_later)
        hipLaunchKernelGGL((distill_kept_kernel<T>), dim3((unsigned)std::min<int64_t>(a.n, 1 << 16)), dim3(64), 4 * record_words(a.k), s, a);
    return hipGetLastError();
}
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) { return a.tail ? launch_backward_as<decltype(t), true>(a, s) : launch_backward_as<decltype(t), false>(a, s); });
}

}  // namespace ens
