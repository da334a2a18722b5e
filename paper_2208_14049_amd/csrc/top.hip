// The k best classes of a row, the lowest class first among equal values, NaN below everything.
//
// Values are compared as 32-bit keys whose order is theirs.  Of the threads' own maxima the k-th largest, t, is a bound: k values at least are no
// smaller.  What is larger than t (some k (1 + k / threads) values where the row is in no order) is collected in LDS and ranked by comparing every pair,
// 32 bits of key before the class.  Where too many are larger the bound is raised by halving its distance to the maximum, and where equal
// ones at the bound are too many the lowest classes among them are found walking the row in order.
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

enum { TOP_VALUE = 0, TOP_LOG = 1, TOP_LOG_SOFTMAX = 2 };
constexpr int TOP_THREADS = 256, TOP_ROOM = 1024;

__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);                 // both zeros are one
    return v != v ? 0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    if (key == 0u) return __uint_as_float(0x7FC00000u);
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

template <int THREADS>
__device__ __forceinline__ int group_count(int v, int* box) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) v += box[w];
    return v;
}

template <class T>
__global__ __launch_bounds__(TOP_THREADS) void top_kernel(const TopArgs a) {
    __shared__ uint64_t found[TOP_ROOM];
    __shared__ uint32_t maxima[TOP_THREADS], bound;
    __shared__ float box[TOP_THREADS / 64];
    __shared__ int ibox[TOP_THREADS / 64], count;
    const int tid = threadIdx.x, k = a.k;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.values + row * a.ld;
        const Row<T, TOP_THREADS> x(p, a.classes);
        uint32_t best = 0;
        float mx = LOWEST;
        x.each(tid, [&](float v, int) { best = max(best, key_of(v)); mx = fmaxf(mx, v); });
        float shift = 0.f;
        if (a.form == TOP_LOG_SOFTMAX) {
            mx = group_max<TOP_THREADS>(mx, box);
            float sum = 0.f;
            x.each(tid, [&](float v, int) { sum += exp_of((v - mx) * a.inv_temperature); });
            sum = group_sum<TOP_THREADS>(sum, box);
            shift = sum == 0.f ? 0.f : logf(sum);               // a row of minus infinities keeps them
        }
        maxima[tid] = best;
        if (tid == 0) count = 0;
        __syncthreads();
        int rank = 0;
        for (int i = 0; i < TOP_THREADS; i++) rank += maxima[i] > best || (maxima[i] == best && i < tid);
        if (rank == k - 1) bound = best;
        if (rank == 0) ibox[0] = (int)best;
        __syncthreads();
        uint32_t t = bound, high = (uint32_t)ibox[0];
        auto larger = [&](uint32_t than) {
            int c = 0;
            x.each(tid, [&](float v, int) { c += key_of(v) > than; });
            return group_count<TOP_THREADS>(c, ibox);
        };
        int above = larger(t);
        if (above > TOP_ROOM) {                                  // k values at least are larger than t, none is larger than high
            while (high - t > 1u) {
                const uint32_t middle = t + (high - t) / 2;
                const int c = larger(middle);
                if (c >= k) t = middle, above = c;
                else high = middle;
                if (c >= k && c <= TOP_ROOM) break;
            }
            if (above > TOP_ROOM) {                              // the k-th value is `high` itself
                t = high;
                above = larger(t);
            }
        }
        int equal = 0;
        x.each(tid, [&](float v, int) { equal += key_of(v) == t; });
        equal = group_count<TOP_THREADS>(equal, ibox);
        const bool all = above + equal <= TOP_ROOM;
        x.each(tid, [&](float v, int c) {
            const uint32_t key = key_of(v);
            if (key > t || (all && key == t)) {
                const int at = atomicAdd(&count, 1);
                found[at] = (uint64_t)key << 32 | (0xFFFFFFFFu - (uint32_t)c);
            }
        });
        __syncthreads();
        int have = count;
        if (!all && above < k) {                                 // the lowest of the equal ones, in order
            for (int c0 = 0; have < k && c0 < a.classes; c0 += TOP_THREADS) {
                const int c = c0 + tid;
                const bool hit = c < a.classes && key_of(up(p[c])) == t;
                const unsigned long long mask = __ballot(hit);
                __syncthreads();
                if ((tid & 63) == 0) ibox[tid >> 6] = __popcll(mask);
                __syncthreads();
                int at = have + __popcll(mask & ((1ull << (tid & 63)) - 1));
                for (int w = 0; w < TOP_THREADS / 64; w++) {
                    if (w < tid >> 6) at += ibox[w];
                    have += ibox[w];
                }
                if (hit && at < k) found[at] = (uint64_t)t << 32 | (0xFFFFFFFFu - (uint32_t)c);
            }
            have = min(have, k);
            __syncthreads();
        }
        for (int i = tid; i < have; i += TOP_THREADS) {
            const uint64_t one = found[i];
            int at = 0;
            for (int o = 0; o < have; o++) at += found[o] > one;
            if (at < k) {
                const float v = value_of((uint32_t)(one >> 32));
                a.index[row * k + at] = (int32_t)(0xFFFFFFFFu - (uint32_t)one);
                a.value[row * k + at] = a.form == TOP_VALUE ? v : a.form == TOP_LOG ? logf(v) : (v - mx) * a.inv_temperature - shift;
            }
        }
        __syncthreads();
    }
}

int64_t top_workspace(int64_t, int, int, int) { return 0; }

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        hipLaunchKernelGGL((top_kernel<decltype(t)>), dim3((unsigned)std::min<int64_t>(a.n, 1 << 16)), dim3(TOP_THREADS), 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace ens
