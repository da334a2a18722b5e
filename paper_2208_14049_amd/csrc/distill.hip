// Distillation: a student's logits x against the classes that a teacher kept of a row, with the logarithms t of their probabilities.
//   p = softmax(x / T);  q = softmax(t) over the kept classes (tail off), or q = e^t and q_0 = max(0, 1 - sum q) for all the others (tail on)
//   loss = T^2 (sum q ln(q / p) [+ q_0 ln(q_0 / p_0)]),  p_0 = sum of p over the classes that were not kept
//   dloss/dx_c = T (S p_c - q_c), S = sum q, and with tail (S = sum q + q_0) for a class that was not kept T (S - q_0 / p_0) p_c
// A class that is listed twice has the sum of its q.  An entry outside the row is not there.  With tail on and p_0 = 0 the tail counts
// nothing.  A row without a kept class of any probability (tail off), or without a finite logit, counts nothing.
//
// With E the sum of e = e^((x - max) / T) over the kept classes and R over the others, Z = E + R: both are summed for themselves, since R as a
// difference would lose what a sure student leaves to the others.  (S - q_0 / p_0) / Z is (sum q - q_0 E / R) / Z.
//
// Bound by memory: a row read, and its gradient written.  A workgroup keeps a row in registers from its maximum through the sums to the gradient, so that
// it is read once (up to 131 072 classes of 16 bits, half as many of fp32), with as many threads as leave the most rows to a compute unit at a time;
// longer rows, and few of the longest, go in parts of 2 048 pieces of 16 bytes, which are read twice.  The teacher's record is read by the first
// wavefront while the others' loads are on their way.
// Gradient with the loss: 4 096 rows of 128 000 bf16 classes 415 us (5.06 TB/s of what has to move; torch's copy of them 437), 1 021 rows of 50 001 with the
// tail 53 us (3.8 TB/s, two rows a compute unit at a time: a quarter of the time goes to their ends), 700 rows of 200 000 180 us (parts).
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

constexpr int KEPT_LANES = DISTILL_MAX_K / 64;
constexpr int CUS = 256;                                         // compute units

// The teacher's record of a row in LDS, as a wavefront leaves it: class (or -1) and q of k entries, the sum of q, q_0, and the sum of q ln q.
struct Record {
    int* index;
    float* q;
    float* sums;
};
__device__ __forceinline__ void read_record(const DistillArgs& a, int64_t row, int lane, const Record& r) {
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
#pragma unroll
    for (int o = 0; o < KEPT_LANES; o++) {
        const int entries = min(64, a.k - 64 * o);
        for (int l = 0; l < entries; l++) {
            const int other = __builtin_amdgcn_readlane(c[o], l);
            int same = 0;
#pragma unroll
            for (int i = 0; i < KEPT_LANES; i++)
                if (64 * i < a.k) same += __popcll(__ballot(c[i] == other));
            twice = twice || (same > 1 && other >= 0);
        }
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
        r.sums[1] = a.tail ? fmaxf(0.f, 1.f - mass) : 0.f;
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

// e of a piece into the sums over kept classes and others
template <int N>
__device__ __forceinline__ void add_piece(const float (&e)[N], uint32_t marked, float& kept, float& others) {
    if (__builtin_expect(__ballot(marked != 0) == 0, 1)) {
        others += sum_of(e);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
        const bool hit = marked >> i & 1;
        kept += hit ? e[i] : 0.f;
        others += hit ? 0.f : e[i];
    }
}

// What multiplies e in the gradient of a class that was not kept, and of one that was.
struct Factors { float other, kept; };
// kept_share: E / Z, over_others: 1 / R or 0 where R is
__device__ __forceinline__ Factors factors(float mass, float rest, float inv_total, float kept_share, float over_others, float weight) {
    const bool with_rest = rest > 0.f && over_others != 0.f;
    return Factors{weight * (mass * inv_total - (with_rest ? rest * kept_share * over_others : 0.f)),
                   weight * (mass + (with_rest ? rest : 0.f)) * inv_total};
}

// LDS of a workgroup: a float for each of 16 wavefronts, the record, the marks
static __host__ __device__ int record_words(int k) { return 16 + 2 * k + 3; }

// A workgroup a row, the row in registers between its maximum, its sums and its gradient.  The registers that a thread may use are stated by the
// wavefronts that are to fit: with 169 instead of 126 a compute unit had one row of 50 001 classes at a time instead of two, 108 us instead of 68.
template <class T, bool TAIL, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS, PIECES == 28 ? 3 : PIECES == 16 ? 4 : PIECES == 8 ? 5 : 6) void distill_held_kernel(const DistillArgs a) {
    extern __shared__ int lds[];
    const int tid = threadIdx.x, k = a.k;
    float* const box = (float*)lds;
    const Record record{lds + 16, (float*)lds + 16 + k, (float*)lds + 16 + 2 * k};
    uint32_t* const marks = (uint32_t*)lds + record_words(k);
    const float cooling = 1.f / a.temperature;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.logits + row * a.ld;
        const Row<T, THREADS> x(p, a.classes);
        Held<T, THREADS, PIECES> held;
        held.load(x, tid);
        if (TAIL)
            for (int i = tid; i < mark_words<T, THREADS>(THREADS * PIECES); i += THREADS) marks[i] = 0;
        if (tid < 64) read_record(a, row, tid, record);
        group_sync<THREADS>();
        float at_kept[(DISTILL_MAX_K + THREADS - 1) / THREADS];
        const int shift = x.HEADS - x.head;
#pragma unroll
        for (int i = 0; i < (DISTILL_MAX_K + THREADS - 1) / THREADS; i++) {
            const int j = tid + i * THREADS, at = j < k ? record.index[j] : -1;
            at_kept[i] = at >= 0 ? up(p[at]) : 0.f;
            if (TAIL && at >= 0) atomicOr(&marks[(at + shift) >> 5], 1u << ((at + shift) & 31));
        }
        const float mx = group_max<THREADS>(held.max(x), box);
        if (TAIL && THREADS == 64) group_sync<THREADS>();
        const Exp power(mx, cooling);
        float kept = 0.f, others = 0.f;
        {
            const float e = power(held.one);
            const bool hit = TAIL && held.at >= 0 && (marks[(held.at + shift) >> 5] >> ((held.at + shift) & 31) & 1);
            if (hit) kept = e;
            else others = e;
        }
        held.each(x, [&](float (&v)[PIECE<T>], int piece) {
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) v[e] = power(v[e]);
            if (TAIL) add_piece(v, piece_marks<T, THREADS>(marks, piece, tid), kept, others);
            else others += sum_of(v);
        });
        others = group_sum<THREADS>(others, box);
        if (TAIL) kept = group_sum<THREADS>(kept, box);
        const float total = others + kept, off = power.off(), ln_total = logf(total * off);
        float cross = 0.f;                                       // sum q ln p
#pragma unroll
        for (int i = 0; i < (DISTILL_MAX_K + THREADS - 1) / THREADS; i++) {
            const int j = tid + i * THREADS;
            if (j < k && record.q[j] != 0.f) cross += record.q[j] * ((at_kept[i] - mx) / a.temperature - ln_total);
        }
        cross = group_sum<THREADS>(cross, box);
        const float mass = record.sums[0], rest = record.sums[1];
        if (tid == 0) {
            const float ln_others = TAIL ? logf(others * off) : NONE;
            float loss = record.sums[2] - cross;
            if (TAIL && rest > 0.f && others != 0.f) loss += rest * (logf(rest) - (ln_others - ln_total));
            a.loss[row] = total == 0.f ? 0.f : loss * a.temperature * a.temperature;
            a.state[row * 3] = mx;
            a.state[row * 3 + 1] = ln_total;
            a.state[row * 3 + 2] = ln_others;
        }
        if (a.d_logits) {
            T* const out = (T*)a.d_logits + row * a.ld_d;
            const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature, inv_total = 1.f / total;
            const bool none = weight == 0.f || total == 0.f;
            const Factors f = factors(mass, TAIL ? rest : 0.f, inv_total, kept * inv_total, others != 0.f ? 1.f / others : 0.f, weight);
            if (none) held.map(x, tid, out, [&](float) { return 0.f; });
            else held.map(x, tid, out, [&](float v) { return f.other * power(v); });
            group_sync<THREADS>();
            if (!none)
#pragma unroll
                for (int i = 0; i < (DISTILL_MAX_K + THREADS - 1) / THREADS; i++) {
                    const int j = tid + i * THREADS;
                    if (j < k && record.index[j] >= 0)
                        out[record.index[j]] = (T)(f.kept * power(at_kept[i]) - weight * record.q[j]);
                }
        }
        group_sync<THREADS>();
    }
}

// The rows in parts, for rows that are too long for a workgroup's registers or too few: first every part's maximum and sums and the logits of the
// kept classes go to the workspace, then every part's workgroup joins them and writes its part of the gradient, the first one the loss.  The second
// step by itself, from the state, is the backward pass.  A part is in registers too.
constexpr int PART_THREADS = 256, PART_PIECES = 8;
struct Parts {
    int parts, length;                                           // of every part but the last
    __host__ __device__ int64_t row_floats(int k) const { return (int64_t)parts * 3 + k; }
};

template <class T, bool TAIL>
__global__ __launch_bounds__(PART_THREADS, 6) void distill_part_kernel(const DistillArgs a, const Parts split) {
    extern __shared__ int lds[];
    const int tid = threadIdx.x, k = a.k;
    float* const box = (float*)lds;
    uint32_t* const marks = (uint32_t*)lds + 16;
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
        for (int j = tid; j < k; j += PART_THREADS) {
            const int64_t at = (int64_t)a.index[row * k + j] - first;
            if (at < 0 || at >= length) continue;
            out[split.parts * 3 + j] = up(p[at]);
            if (TAIL) atomicOr(&marks[(at + shift) >> 5], 1u << ((at + shift) & 31));
        }
        const float mx = group_max<PART_THREADS>(held.max(x), box);
        const Exp power(mx, cooling);
        float kept = 0.f, others = 0.f;
        {
            const float e = power(held.one);
            if (TAIL && held.at >= 0 && (marks[(held.at + shift) >> 5] >> ((held.at + shift) & 31) & 1)) kept = e;
            else others = e;
        }
        held.each(x, [&](float (&v)[PIECE<T>], int piece) {
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) v[e] = power(v[e]);
            if (TAIL) add_piece(v, piece_marks<T, PART_THREADS>(marks, piece, tid), kept, others);
            else others += sum_of(v);
        });
        others = group_sum<PART_THREADS>(others, box) * power.off();
        if (TAIL) kept = group_sum<PART_THREADS>(kept, box) * power.off();
        if (tid == 0) {
            out[part * 3] = mx;
            out[part * 3 + 1] = kept;
            out[part * 3 + 2] = others;
        }
        __syncthreads();
    }
}

template <class T, bool TAIL, bool JOIN, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS, 6) void distill_gradient_kernel(const DistillArgs a, const Parts split) {
    extern __shared__ int lds[];
    __shared__ float found[4];
    constexpr int KEPT = (DISTILL_MAX_K + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, k = a.k;
    const Record record{lds + 16, (float*)lds + 16 + k, (float*)lds + 16 + 2 * k};
    const float cooling = 1.f / a.temperature;
    const int per_row = a.d_logits ? split.parts : 1;            // the first part alone has the loss
    for (int64_t job = blockIdx.x; job < a.n * per_row; job += gridDim.x) {
        const int64_t row = job / per_row;
        const int part = (int)(job - row * per_row), first = part * split.length, length = min(split.length, a.classes - first);
        const float* const from = (const float*)a.workspace + row * split.row_floats(k);
        const T* const p = (const T*)a.logits + row * a.ld + first;
        const Row<T, THREADS> x(p, length);
        Held<T, THREADS, PIECES> held;
        if (a.d_logits) held.load(x, tid);
        if (tid < 64) {
            read_record(a, row, lane, record);
            if (JOIN) {
                float m = LOWEST, kept = 0.f, others = 0.f;
                for (int i = lane; i < split.parts; i += 64) m = fmaxf(m, from[i * 3]);
                m = lanes_max(m);
                for (int i = lane; i < split.parts; i += 64) {
                    const Exp power(m, cooling);
                    const float less = __builtin_amdgcn_exp2f((from[i * 3] - m) * power.c);
                    kept += from[i * 3 + 1] * less;
                    others += from[i * 3 + 2] * less;
                }
                kept = lanes_sum(kept);
                others = lanes_sum(others);
                if (lane == 0) {
                    found[0] = m;
                    found[1] = kept + others;
                    found[2] = kept;
                    found[3] = others;
                }
                if (part == 0) {
                    const float ln_total = logf(kept + others);
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    float cross = 0.f;
                    for (int j = lane; j < k; j += 64)
                        if (record.q[j] != 0.f) cross += record.q[j] * ((from[split.parts * 3 + j] - m) / a.temperature - ln_total);
                    cross = lanes_sum(cross);
                    if (lane == 0) {
                        const float rest = record.sums[1], ln_others = TAIL ? logf(others) : NONE;
                        float loss = record.sums[2] - cross;
                        if (TAIL && rest > 0.f && others != 0.f) loss += rest * (logf(rest) - (ln_others - ln_total));
                        a.loss[row] = kept + others == 0.f ? 0.f : loss * a.temperature * a.temperature;
                        a.state[row * 3] = m;
                        a.state[row * 3 + 1] = ln_total;
                        a.state[row * 3 + 2] = ln_others;
                    }
                }
            }
        }
        group_sync<THREADS>();
        if (a.d_logits) {
            T* const out = (T*)a.d_logits + row * a.ld_d + first;
            const float mass = record.sums[0], rest = TAIL ? record.sums[1] : 0.f;
            const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature;
            float mx, total;
            Factors f;
            if (JOIN) {
                mx = found[0];
                total = found[1];
                f = factors(mass, rest, 1.f / total, found[2] / total, found[3] != 0.f ? 1.f / found[3] : 0.f, weight);
            } else {
                mx = a.state[row * 3];
                const float ln_total = a.state[row * 3 + 1], ln_others = a.state[row * 3 + 2];
                total = expf(ln_total);
                const bool others = TAIL && ln_others > NONE;
                f = factors(mass, others ? rest : 0.f, 1.f / total, others ? -expm1f(ln_others - ln_total) : 0.f, others ? expf(-ln_others) : 0.f, weight);
            }
            const bool none = weight == 0.f || total == 0.f;
            float at_kept[KEPT];
            int at[KEPT];
#pragma unroll
            for (int i = 0; i < KEPT; i++) {
                const int j = tid + i * THREADS;
                const int64_t here = j < k && record.index[j] >= 0 ? (int64_t)record.index[j] - first : -1;
                at[i] = here >= 0 && here < length ? (int)here : -1;
                at_kept[i] = at[i] < 0 ? 0.f : JOIN ? from[split.parts * 3 + j] : up(p[at[i]]);
            }
            group_sync<THREADS>();                               // out may be p
            const Exp power(mx, cooling);
            const float other = f.other * power.off(), own = f.kept * power.off();
            if (none) held.map(x, tid, out, [&](float) { return 0.f; });
            else held.map(x, tid, out, [&](float v) { return other * power(v); });
            group_sync<THREADS>();
            if (!none)
#pragma unroll
                for (int i = 0; i < KEPT; i++)
                    if (at[i] >= 0) out[at[i]] = (T)(own * power(at_kept[i]) - weight * record.q[tid + i * THREADS]);
        }
        group_sync<THREADS>();
    }
}

// Parts as long as a workgroup holds, or some 1 024 of them, of 4 096 classes at least.
static Parts split_rows(int64_t n, int classes, int dtype) {
    const int64_t piece = dtype == 0 ? 4 : 8, most = (classes + 4095) / 4096, want = std::max<int64_t>(1, 1024 / n);
    const int parts = (int)std::max<int64_t>((classes / piece + PART_THREADS * PART_PIECES - 1) / (PART_THREADS * PART_PIECES), std::min(most, want));
    if (parts <= 1) return Parts{1, classes};
    int length = ((classes + parts - 1) / parts + 63) / 64 * 64;
    length = std::min<int>(length, PART_THREADS * PART_PIECES * piece);
    return Parts{(classes + length - 1) / length, length};
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
    const int lds = 4 * (16 + (TAIL ? mark_words<T, PART_THREADS>(PART_THREADS * PART_PIECES) : 0));
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
        hipLaunchKernelGGL((distill_gradient_kernel<T, TAIL, false, 64, 4>), rows, dim3(64), 4 * record_words(a.k), s, a, Parts{1, a.classes});
        return hipGetLastError();
    }
    const Parts split = split_rows(a.n, a.classes, a.dtype);
    const dim3 grid((unsigned)std::min<int64_t>(a.n * split.parts, 1 << 16));
    hipLaunchKernelGGL((distill_gradient_kernel<T, TAIL, false, PART_THREADS, PART_PIECES>), grid, dim3(PART_THREADS), 4 * record_words(a.k), s, a, split);
    return hipGetLastError();
}
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) { return a.tail ? launch_backward_as<decltype(t), true>(a, s) : launch_backward_as<decltype(t), false>(a, s); });
}

}  // namespace ens
