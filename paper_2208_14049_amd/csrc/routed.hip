// Combination with weights of each row: y_c = sum_j w_j p_j(c), p_j the softmax of the j-th chosen member's logits.  Members that a row
// did not choose are not read.  A choice outside the members is not there, one that comes twice counts with the sum of its weights.  A member's row of
// minus infinities gives nothing.
//   backward: dL/dw_j = sum_c g_c p_j(c);  dL/dz_j(c) = W p_j(c) (g_c - dL/dw_j), W the weights of that member in the row
//
// Bound by memory: k rows read and one written, and backward k + 1 read and one for each member written.  Rows are in registers from their
// maximum to the last use of their values, and the sum over members too, so that each is read once.  A wavefront takes a row of up to 256 pieces of 16
// bytes, a workgroup one of up to 8 192 (backward 4 096); longer ones are walked in memory: forward for the maximum, for the sum and class by class, backward twice.
// 8 100 rows of 1 000 fp32 classes, three of twelve members: 27 us (4.8 TB/s, as calls without a profiler 26: at the rate of memory).  1 023 rows of 32 001 bf16,
// two of four members: 76 us forward among the backward passes (3.4 TB/s; 66 by itself over four sets of inputs), 116 us backward with the gradients of weights
// and logits (4.5 TB/s; rows of odd length, two at a time a compute unit).  64 000 classes: 159 and 275 us.  Long ones are far from memory's rate: 2 048 rows of
// 128 000 1 008 us forward (2.1 TB/s of what has to move, read three times) and 1 005 backward (4.2); one such row, by one workgroup, 70 and 18.
// The accumulators of 16-bit rows fill the registers: 4 are spilled with 512 threads (backward too), 17 with 1 024.
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

// A row's choices, one a lane, the same in every wavefront: the member or -1, and its weight.
struct Choices {
    int member;
    float weight;
    uint64_t left;                                               // choices to be taken
    __device__ __forceinline__ Choices(const RoutedArgs& a, int64_t row, int lane) {
        const int64_t at = row * a.k + lane;
        member = lane < a.k ? a.chosen[at] : -1;
        if (member >= a.members) member = -1;
        weight = member >= 0 ? a.weights[at] : 0.f;
        left = __ballot(member >= 0);
    }
    // zeros where a choice is not there
    __device__ __forceinline__ void clear_state(const RoutedArgs& a, int64_t row, int tid) const {
        if (a.state && tid < a.k && member < 0) a.state[(row * a.k + tid) * 2] = a.state[(row * a.k + tid) * 2 + 1] = 0.f;
    }
    __device__ __forceinline__ uint64_t of(int m) const { return __ballot(member == m); }
    // weights of the choices in the mask, in order
    __device__ __forceinline__ float sum(uint64_t mask) const {
        float w = 0.f;
        for (; mask; mask &= mask - 1) w += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), __builtin_ctzll(mask)));
        return w;
    }
};

template <class T, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS, 4) void combine_routed_kernel(const RoutedArgs a) {
    __shared__ float box[16];
    const int tid = threadIdx.x, lane = tid & 63, classes = a.classes;
    const Uncut<PIECE<T>> cut(classes);                          // (cut in lines of the output there were too few registers: 61 us became 75)
    const int one = cut.single(tid);
    const bool past = a.n * classes >= 16 << 20;                 // 64 MiB: smaller outputs are in the caches for what reads them next
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        Choices choices(a, row, lane);
        float y[PIECES][PIECE<T>], y_one = 0.f;
#pragma unroll
        for (int i = 0; i < PIECES; i++)
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) y[i][e] = 0.f;
        while (choices.left) {
            const int m = __builtin_amdgcn_readlane(choices.member, __builtin_ctzll(choices.left));
            const uint64_t same = choices.of(m);
            choices.left &= ~same;
            Span<T, THREADS, PIECES> z;
            z.load((const T*)a.logits[m] + row * a.ld, cut, tid);
            float mx = fmaxf(LOWEST, z.one), sum = 0.f;
            z.each(cut, [&](const float (&v)[PIECE<T>], int) {
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) mx = fmaxf(mx, v[e]);
            });
            mx = group_max<THREADS>(mx, box);
            const Exp power(mx, 1.f);
            z.each(cut, [&](float (&v)[PIECE<T>], int) {
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) v[e] = power(v[e]);
                sum += sum_of(v);
            });
            const float e_one = power(z.one);
            sum = group_sum<THREADS>(sum + e_one, box);
            if (a.state && tid < 64 && same >> lane & 1) {
                a.state[(row * a.k + lane) * 2] = mx;
                a.state[(row * a.k + lane) * 2 + 1] = logf(sum * power.off());
            }
            const float share = sum == 0.f ? 0.f : choices.sum(same) / sum;
            y_one = fmaf(share, e_one, y_one);
            z.each(cut, [&](const float (&v)[PIECE<T>], int i) {
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) y[i][e] = fmaf(share, power(v[e]), y[i][e]);
            });
        }
        float* const out = a.probs + row * classes;
        if (one >= 0) out[one] = y_one;
#pragma unroll
        for (int i = 0; i < PIECES; i++)
            if (tid < cut.pieces - i * THREADS) store_floats(out + cut.head + (i * THREADS + tid) * PIECE<T>, y[i], past);
        choices.clear_state(a, row, tid);
    }
}

// A row by a workgroup in memory: the maxima and sums of all chosen members first, then class by class.
constexpr int LONG_THREADS = 1024;
template <class T>
__global__ __launch_bounds__(LONG_THREADS) void combine_routed_long_kernel(const RoutedArgs a) {
    __shared__ float box[16], top[ROUTED_MAX_K], part[ROUTED_MAX_K];
    const int tid = threadIdx.x, lane = tid & 63;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        Choices choices(a, row, lane);
        choices.clear_state(a, row, tid);
        uint64_t firsts = 0;
        while (choices.left) {
            const int j = __builtin_ctzll(choices.left), m = __builtin_amdgcn_readlane(choices.member, j);
            const uint64_t same = choices.of(m);
            choices.left &= ~same;
            firsts |= 1ull << j;
            const Row<T, LONG_THREADS> z((const T*)a.logits[m] + row * a.ld, a.classes);
            float mx = LOWEST, sum = 0.f;
            z.each(tid, [&](float v, int) { mx = fmaxf(mx, v); });
            mx = group_max<LONG_THREADS>(mx, box);
            const Exp power(mx, 1.f);
            z.each(tid, [&](float v, int) { sum += power(v); });
            sum = group_sum<LONG_THREADS>(sum, box);
            if (a.state && tid < 64 && same >> lane & 1) {
                a.state[(row * a.k + lane) * 2] = mx;
                a.state[(row * a.k + lane) * 2 + 1] = logf(sum * power.off());
            }
            if (tid == 0) {
                top[j] = mx;
                part[j] = sum == 0.f ? 0.f : choices.sum(same) / sum;
            }
        }
        __syncthreads();
        for (int c = tid; c < a.classes; c += LONG_THREADS) {
            float y = 0.f;
            for (uint64_t left = firsts; left; left &= left - 1) {
                const int j = __builtin_ctzll(left), m = __builtin_amdgcn_readlane(choices.member, j);
                y = fmaf(part[j], Exp(top[j], 1.f)(up(((const T*)a.logits[m] + row * a.ld)[c])), y);
            }
            a.probs[row * (int64_t)a.classes + c] = y;
        }
        __syncthreads();
    }
}

// What multiplies the terms of a member's row in its softmax: 1 / sum, 0 for a row that holds nothing.
__device__ __forceinline__ float inverse_sum(const Exp& power, float ln_sum) { return ln_sum == NONE ? 0.f : expf(-ln_sum) * power.off(); }

// A job is a row and a member (BY_MEMBER: the member's gradient, zeros where the row did not choose it) or a row and a choice (the weights'
// gradients alone).  A workgroup of a long row has one, and the jobs of a row go to one XCD, one after the other, so that the row of g is read from memory
// once; a wavefront takes all the jobs of a row of one piece a lane (8 100 rows of 10 classes, three of twelve members: 15 us instead of 30, as a call from
// Python; of 1 000 classes 93 instead of 87).
template <class T, int THREADS, int PIECES, bool BY_MEMBER>
__global__ __launch_bounds__(THREADS, PIECES == 8 ? 4 : 5) void combine_routed_backward_kernel(const RoutedArgs a, const int64_t jobs) {
    __shared__ float box[16];
    const int tid = threadIdx.x, lane = tid & 63, classes = a.classes;
    const int per_row = BY_MEMBER ? a.members : a.k;
    auto one_job = [&](const int64_t row, const Choices& choices, const int what) {
        const int m = BY_MEMBER ? what : __builtin_amdgcn_readlane(choices.member, what);
        if (a.d_weights && what == 0 && tid < a.k && choices.member < 0) a.d_weights[row * a.k + tid] = 0.f;
        const uint64_t same = m < 0 ? 0 : choices.of(m);
        T* const out = BY_MEMBER && a.d_logits[m] ? (T*)a.d_logits[m] + row * a.ld_d : nullptr;
        const Cut<PIECE<T>, THREADS> cut(out ? out : (const T*)a.logits[m < 0 ? 0 : m] + row * a.ld, sizeof(T), classes);
        const int one = cut.single(tid), pieces = cut.pieces;
        if (!same || (!BY_MEMBER && __builtin_ctzll(same) != what)) {
            if (!out) return;
            if (one >= 0) out[one] = (T)0.f;
            for (int i = tid; i < pieces; i += THREADS) store_past(out + cut.head + (int64_t)i * PIECE<T>, make_uint4(0, 0, 0, 0));
            return;
        }
        const int j = __builtin_ctzll(same);
        const T* const z_row = (const T*)a.logits[m] + row * a.ld;
        const float* const g_row = a.d_probs + row * classes;
        const float mx = a.state[(row * a.k + j) * 2], ln_sum = a.state[(row * a.k + j) * 2 + 1];
        const Exp power(mx, 1.f);
        const float inverse = inverse_sum(power, ln_sum), weight = choices.sum(same);
        float dot = 0.f;
        if constexpr (PIECES > 0) {
            Span<T, THREADS, PIECES> z;
            float g[PIECES][PIECE<T>], g_one = one >= 0 ? g_row[one] : 0.f;
            z.load(z_row, cut, tid);
#pragma unroll
            for (int i = 0; i < PIECES; i++) {
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) g[i][e] = 0.f;
                if (tid < pieces - i * THREADS) load_floats(g_row + cut.head + (i * THREADS + tid) * PIECE<T>, g[i]);
            }
            z.each(cut, [&](const float (&v)[PIECE<T>], int i) {
                float t[PIECE<T>];
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) t[e] = power(v[e]) * g[i][e];
                dot += sum_of(t);
            });
            dot = group_sum<THREADS>(dot + power(z.one) * g_one, box) * inverse;
            if (out) {
                const float scale = weight * inverse;
                if (one >= 0) out[one] = (T)(scale * power(z.one) * (g_one - dot));
                z.each(cut, [&](float (&v)[PIECE<T>], int i) {
                    if (tid >= pieces - i * THREADS) return;
#pragma unroll
                    for (int e = 0; e < PIECE<T>; e++) v[e] = scale * power(v[e]) * (g[i][e] - dot);
                    store_past((char*)(out + cut.head + i * THREADS * PIECE<T>) + (uint32_t)tid * 16u, pack(v, out));
                });
            }
        } else {
            auto walk = [&](auto f) {
                if (one >= 0) {
                    const float v[1] = {up(z_row[one])}, g[1] = {g_row[one]};
                    f(v[0], g[0], one);
                }
                for (int64_t i = tid; i < pieces; i += THREADS) {
                    float v[PIECE<T>], g[PIECE<T>];
                    unpack(load_loose(z_row + cut.head + i * PIECE<T>), v, z_row);
                    load_floats(g_row + cut.head + i * PIECE<T>, g);
#pragma unroll
                    for (int e = 0; e < PIECE<T>; e++) f(v[e], g[e], cut.head + i * PIECE<T> + e);
                }
            };
            walk([&](float v, float g, int64_t) { dot = fmaf(power(v), g, dot); });
            dot = group_sum<THREADS>(dot, box) * inverse;
            const float scale = weight * inverse;
            if (out) walk([&](float v, float g, int64_t c) { out[c] = (T)(scale * power(v) * (g - dot)); });
        }
        if (a.d_weights && tid < 64 && same >> lane & 1) a.d_weights[row * a.k + lane] = dot;
    };
    if constexpr (PIECES == 1) {
        for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
            const Choices choices(a, row, lane);
            for (int what = 0; what < per_row; what++) one_job(row, choices, what);
        }
    } else {
        for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
            const int64_t eights = job / 8, row = eights / per_row * 8 + job % 8;
            if (row < a.n) one_job(row, Choices(a, row, lane), (int)(eights % per_row));
        }
    }
}

hipError_t launch_combine_routed(const RoutedArgs& a, hipStream_t s) {
    return by_type(a.dtype, [&](auto t) {
        typedef decltype(t) T;
        const int pieces = (a.classes + PIECE<T> - 1) / PIECE<T>;
        const dim3 rows((unsigned)std::min<int64_t>(a.n, 1 << 16));
        if (pieces <= 64) hipLaunchKernelGGL((combine_routed_kernel<T, 64, 1>), rows, dim3(64), 0, s, a);
        else if (pieces <= 64 * 4) hipLaunchKernelGGL((combine_routed_kernel<T, 64, 4>), rows, dim3(64), 0, s, a);
        else if (pieces <= 256 * 4) hipLaunchKernelGGL((combine_routed_kernel<T, 256, 4>), rows, dim3(256), 0, s, a);
        else if (pieces <= 512 * 8) hipLaunchKernelGGL((combine_routed_kernel<T, 512, 8>), rows, dim3(512), 0, s, a);
        else if (pieces <= 1024 * 8) hipLaunchKernelGGL((combine_routed_kernel<T, 1024, 8>), rows, dim3(1024), 0, s, a);
        else hipLaunchKernelGGL((combine_routed_long_kernel<T>), rows, dim3(LONG_THREADS), 0, s, a);
        return hipGetLastError();
    });
}

template <class T, bool BY_MEMBER>
static hipError_t launch_backward(const RoutedArgs& a, hipStream_t s) {
    const int pieces = (a.classes + PIECE<T> - 1) / PIECE<T>;
    const int64_t jobs = (a.n + 7) / 8 * 8 * (BY_MEMBER ? a.members : a.k);
    const dim3 grid((unsigned)std::min<int64_t>(jobs, 1 << 20));
    const dim3 rows((unsigned)std::min<int64_t>(a.n, 1 << 16));
    if (pieces <= 64) hipLaunchKernelGGL((combine_routed_backward_kernel<T, 64, 1, BY_MEMBER>), rows, dim3(64), 0, s, a, jobs);
    else if (pieces <= 64 * 4) hipLaunchKernelGGL((combine_routed_backward_kernel<T, 64, 4, BY_MEMBER>), grid, dim3(64), 0, s, a, jobs);
    else if (pieces <= 256 * 4) hipLaunchKernelGGL((combine_routed_backward_kernel<T, 256, 4, BY_MEMBER>), grid, dim3(256), 0, s, a, jobs);
    else if (pieces <= 512 * 8) hipLaunchKernelGGL((combine_routed_backward_kernel<T, 512, 8, BY_MEMBER>), grid, dim3(512), 0, s, a, jobs);
    else hipLaunchKernelGGL((combine_routed_backward_kernel<T, LONG_THREADS, 0, BY_MEMBER>), grid, dim3(LONG_THREADS), 0, s, a, jobs);
    return hipGetLastError();
}

hipError_t launch_combine_routed_backward(const RoutedArgs& a, hipStream_t s) {
    bool any = false;
    for (int m = 0; m < a.members; m++) any = any || a.d_logits[m];
    return by_type(a.dtype, [&](auto t) { return any ? launch_backward<decltype(t), true>(a, s) : launch_backward<decltype(t), false>(a, s); });
}

}  // namespace ens
