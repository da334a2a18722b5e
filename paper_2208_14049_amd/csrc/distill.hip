// Distillation: a student's logits x against the classes that a teacher kept of a row, with the logarithms t of their probabilities.
//   p = softmax(x / T);  q = softmax(t) over the kept classes (tail off), or q = e^t and q_0 = max(0, 1 - sum q) for all the others (tail on)
//   loss = T^2 (sum q ln(q / p) [+ q_0 ln(q_0 / p_0)]),  p_0 = sum of p over the classes that were not kept
//   dloss/dx_c = T (S p_c - q_c), S = sum q, and with tail (S = sum q + q_0) for a class that was not kept T (S - q_0 / p_0) p_c
// A class that is listed twice has the sum of its q.  An entry outside the row is not there.  With tail on and p_0 = 0 the tail counts
// nothing.  A row without a kept class of any probability (tail off), or without a finite logit, counts nothing.
//
// With E the sum of e = e^((x - max) / T) over the kept classes and R over the others, Z = E + R: both are summed for themselves, since R as a
// difference would lose what a sure student leaves to the others.  (S - q_0 / p_0) / Z is (sum q - q_0 E / R) / Z.
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

constexpr int DISTILL_THREADS = 256;

// The teacher's record of a row, in LDS.  A wavefront reads it: entry j's class or -1, its q, and of them sum and rest.
struct Record {
    int* index;                  // k
    float* q;                    // k
    float* sums;                 // sum of q, q_0, q ln q of all entries and q_0
};
__device__ __forceinline__ void read_record(const DistillArgs& a, int64_t row, int lane, const Record& r) {
    const int32_t* const index = a.index + row * a.k;
    const float* const log_probs = a.log_probs + row * a.k;
    float top = NONE;
    if (!a.tail) {
        for (int j = lane; j < a.k; j += 64)
            if (index[j] >= 0 && index[j] < a.classes) top = fmaxf(top, log_probs[j]);
        top = lanes_max(top);
    }
    float sum = 0.f;
    for (int j = lane; j < a.k; j += 64) {
        const int c = index[j];
        const bool here = c >= 0 && c < a.classes;
        const float t = here ? log_probs[j] : NONE;
        const float q = t == NONE ? 0.f : expf(a.tail ? t : t - top);
        r.index[j] = here ? c : -1;
        r.q[j] = q;
        sum += q;
    }
    sum = lanes_sum(sum);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const float scale = a.tail || sum == 0.f ? 1.f : 1.f / sum;
    // the first entry of a class takes what the later ones have
    for (int j0 = 0; j0 < a.k; j0 += 64) {
        const int j = j0 + lane;
        float q = 0.f;
        int c = -1;
        if (j < a.k) {
            c = r.index[j];
            bool first = true;
            for (int i = 0; i < a.k; i++) {
                const int other = r.index[i];
                if (other == c) {
                    if (i < j) first = false;
                    q += r.q[i];
                }
            }
            if (!first) c = -2;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (j < a.k) {
            r.index[j + a.k] = c < 0 ? -1 : c;
            r.q[j + a.k] = c < 0 ? 0.f : q * scale;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float mass = 0.f, entropy = 0.f;
    for (int j = lane; j < a.k; j += 64) {
        const float q = r.q[j + a.k];
        mass += q;
        if (q != 0.f) entropy += q * logf(q);
    }
    mass = lanes_sum(mass);
    entropy = lanes_sum(entropy);
    const float rest = a.tail ? fmaxf(0.f, 1.f - mass) : 0.f;
    if (lane == 0) {
        r.sums[0] = mass;
        r.sums[1] = rest;
        r.sums[2] = entropy;
    }
}

// LDS: the record twice (as read, and with equal classes joined), three sums, a float for each wavefront; a bit for each class (tail)
static __host__ __device__ int distill_lds(int k, int classes, bool tail) {
    return (4 * k + 3 + DISTILL_THREADS / 64) * 4 + (tail ? (classes + 31) / 32 * 4 : 0);
}

template <class T, bool TAIL, bool BACKWARD>
__global__ __launch_bounds__(DISTILL_THREADS) void distill_kernel(const DistillArgs a) {
    extern __shared__ int lds[];
    const int tid = threadIdx.x, lane = tid & 63, k = a.k;
    const Record record{lds, (float*)lds + 2 * k, (float*)lds + 4 * k};
    float* const box = (float*)lds + 4 * k + 3;
    uint32_t* const marks = (uint32_t*)(box + DISTILL_THREADS / 64);
    const int* const index = record.index + k;
    const float* const q = record.q + k;
    const float inv_t = 1.f / a.temperature;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.logits + row * a.ld;
        const Row<T, DISTILL_THREADS> x(p, a.classes);
        if (tid < 64) read_record(a, row, lane, record);
        if (TAIL && !BACKWARD)
            for (int i = tid; i < (a.classes + 31) / 32; i += DISTILL_THREADS) marks[i] = 0;
        __syncthreads();
        if (TAIL && !BACKWARD) {
            for (int j = tid; j < k; j += DISTILL_THREADS)
                if (index[j] >= 0) atomicOr(&marks[index[j] >> 5], 1u << (index[j] & 31));
            __syncthreads();
        }
        const float mass = record.sums[0], rest = record.sums[1];
        float mx = LOWEST, total = 0.f, others = 0.f, ln_total, ln_others = NONE;
        if constexpr (!BACKWARD) {
            x.each(tid, [&](float v, int) { mx = fmaxf(mx, v); });
            mx = group_max<DISTILL_THREADS>(mx, box);
            float kept = 0.f;
            x.each(tid, [&](float v, int c) {
                const float e = exp_of((v - mx) * inv_t);
                if (TAIL && (marks[c >> 5] >> (c & 31) & 1)) kept += e;
                else others += e;
            });
            others = group_sum<DISTILL_THREADS>(others, box);
            total = others;
            if (TAIL) total += group_sum<DISTILL_THREADS>(kept, box);
            ln_total = logf(total);
            if (TAIL) ln_others = logf(others);
            // sum q ln q - sum q ln p
            float cross = 0.f;
            for (int j = tid; j < k; j += DISTILL_THREADS)
                if (index[j] >= 0 && q[j] != 0.f) cross += q[j] * ((up(p[index[j]]) - mx) * inv_t - ln_total);
            cross = group_sum<DISTILL_THREADS>(cross, box);
            if (tid == 0) {
                float loss = record.sums[2] - cross;
                if (TAIL && rest > 0.f && others != 0.f) loss += rest * (logf(rest) - (ln_others - ln_total));
                a.loss[row] = total == 0.f ? 0.f : loss * a.temperature * a.temperature;
                a.state[row * 3] = mx;
                a.state[row * 3 + 1] = ln_total;
                a.state[row * 3 + 2] = ln_others;
            }
        } else {
            mx = a.state[row * 3];
            ln_total = a.state[row * 3 + 1];
            ln_others = a.state[row * 3 + 2];
        }
        if (BACKWARD || a.d_logits) {
            T* const out = (T*)a.d_logits + row * a.ld_d;
            const float weight = (a.row_weights ? a.row_weights[row] : 1.f) * a.temperature;
            const bool none = weight == 0.f || ln_total == NONE;
            const bool with_rest = TAIL && rest > 0.f && ln_others > NONE;
            const float all = mass + (with_rest ? rest : 0.f);
            // ln(Z / R) beyond 80 belongs to classes of e^-80 and less
            const float factor = with_rest ? mass - rest * expm1f(fminf(ln_total - ln_others, 80.f)) : mass;
            float at_kept[(DISTILL_MAX_K + DISTILL_THREADS - 1) / DISTILL_THREADS];
#pragma unroll
            for (int i = 0; i < (DISTILL_MAX_K + DISTILL_THREADS - 1) / DISTILL_THREADS; i++) {
                const int j = tid + i * DISTILL_THREADS;
                at_kept[i] = j < k && index[j] >= 0 ? up(p[index[j]]) : 0.f;
            }
            __syncthreads();                                     // out may be p
            x.map(tid, out, [&](float v, int) { return none ? 0.f : weight * factor * exp_of((v - mx) * inv_t - ln_total); });
            __syncthreads();
            if (!none)
#pragma unroll
                for (int i = 0; i < (DISTILL_MAX_K + DISTILL_THREADS - 1) / DISTILL_THREADS; i++) {
                    const int j = tid + i * DISTILL_THREADS;
                    if (j < k && index[j] >= 0) out[index[j]] = (T)(weight * (all * exp_of((at_kept[i] - mx) * inv_t - ln_total) - q[j]));
                }
        }
        __syncthreads();
    }
}

int64_t distill_workspace(int64_t, int, int, int) { return 0; }

template <bool BACKWARD>
static hipError_t launch(const DistillArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 16)), group(DISTILL_THREADS);
        const int lds = distill_lds(a.k, a.classes, a.tail && !BACKWARD);
        if (a.tail) hipLaunchKernelGGL((distill_kernel<decltype(t), true, BACKWARD>), grid, group, lds, s, a);
        else hipLaunchKernelGGL((distill_kernel<decltype(t), false, BACKWARD>), grid, group, lds, s, a);
        return hipGetLastError();
    });
}
hipError_t launch_distill(const DistillArgs& a, hipStream_t s) { return launch<false>(a, s); }
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) { return launch<true>(a, s); }

}  // namespace ens
