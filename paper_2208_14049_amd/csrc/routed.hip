// Combination with weights of each row: y_c = sum_j w_j p_j(c), p_j the softmax of the j-th chosen member's logits.  Members that a row
// did not choose are not read.  A choice outside the members is not there.  A member's row of minus infinities gives nothing.
//   backward: dL/dw_j = sum_c g_c p_j(c);  dL/dz_j(c) = W p_j(c) (g_c - dL/dw_j), W the weights of that member in the row
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

constexpr int ROUTED_THREADS = 256;

template <class T>
__global__ __launch_bounds__(ROUTED_THREADS) void combine_routed_kernel(const RoutedArgs a) {
    __shared__ float box[2 * ROUTED_THREADS / 64], top[ROUTED_MAX_K], part[ROUTED_MAX_K];
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const int32_t* const chosen = a.chosen + row * a.k;
        for (int j = 0; j < a.k; j++) {
            const int m = chosen[j];
            if (m < 0 || m >= a.members) continue;
            const Row<T, ROUTED_THREADS> z((const T*)a.logits[m] + row * a.ld, a.classes);
            float mx = LOWEST, sum = 0.f;
            z.each(tid, [&](float v, int) { mx = fmaxf(mx, v); });
            mx = group_max<ROUTED_THREADS>(mx, box);
            z.each(tid, [&](float v, int) { sum += exp_of(v - mx); });
            sum = group_sum<ROUTED_THREADS>(sum, box);
            if (tid == 0) {
                top[j] = mx;
                part[j] = sum == 0.f ? 0.f : a.weights[row * a.k + j] / sum;
                if (a.state) {
                    a.state[(row * a.k + j) * 2] = mx;
                    a.state[(row * a.k + j) * 2 + 1] = logf(sum);
                }
            }
        }
        __syncthreads();
        for (int c = tid; c < a.classes; c += ROUTED_THREADS) {
            float y = 0.f;
            for (int j = 0; j < a.k; j++) {
                const int m = chosen[j];
                if (m < 0 || m >= a.members) continue;
                y = fmaf(part[j], exp_of(up(((const T*)a.logits[m] + row * a.ld)[c]) - top[j]), y);
            }
            a.probs[row * a.classes + c] = y;
        }
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(ROUTED_THREADS) void combine_routed_backward_kernel(const RoutedArgs a) {
    __shared__ float box[2 * ROUTED_THREADS / 64], dot[ROUTED_MAX_K];
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const int32_t* const chosen = a.chosen + row * a.k;
        const float* const g = a.d_probs + row * a.classes;
        const float* const state = a.state + row * a.k * 2;
        for (int j = 0; j < a.k; j++) {
            const int m = chosen[j];
            float d = 0.f;
            if (m >= 0 && m < a.members) {
                const T* const z = (const T*)a.logits[m] + row * a.ld;
                const float mx = state[2 * j], ln = state[2 * j + 1];
                if (ln > NONE || !(ln <= 0.f))
                    for (int c = tid; c < a.classes; c += ROUTED_THREADS) d = fmaf(g[c], exp_of(up(z[c]) - mx - ln), d);
                d = group_sum<ROUTED_THREADS>(d, box);
            }
            if (tid == 0) {
                dot[j] = d;
                if (a.d_weights) a.d_weights[row * a.k + j] = d;
            }
        }
        __syncthreads();
        for (int m = 0; m < a.members; m++) {
            if (!a.d_logits[m]) continue;
            T* const out = (T*)a.d_logits[m] + row * a.ld_d;
            const T* const z = (const T*)a.logits[m] + row * a.ld;
            float weight = 0.f;
            int first = -1;
            for (int j = 0; j < a.k; j++)
                if (chosen[j] == m) {
                    weight += a.weights[row * a.k + j];
                    if (first < 0) first = j;
                }
            const float mx = first >= 0 ? state[2 * first] : 0.f, ln = first >= 0 ? state[2 * first + 1] : 0.f;
            const bool none = first < 0 || (ln <= 0.f && !(ln > NONE));
            for (int c = tid; c < a.classes; c += ROUTED_THREADS)
                out[c] = (T)(none ? 0.f : weight * exp_of(up(z[c]) - mx - ln) * (g[c] - dot[first]));
        }
        __syncthreads();
    }
}

static unsigned routed_blocks(int64_t n) { return (unsigned)std::min<int64_t>(n, 1 << 16); }

hipError_t launch_combine_routed(const RoutedArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        hipLaunchKernelGGL((combine_routed_kernel<decltype(t)>), dim3(routed_blocks(a.n)), dim3(ROUTED_THREADS), 0, s, a);
        return hipGetLastError();
    });
}

hipError_t launch_combine_routed_backward(const RoutedArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        hipLaunchKernelGGL((combine_routed_backward_kernel<decltype(t)>), dim3(routed_blocks(a.n)), dim3(ROUTED_THREADS), 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace ens
