// Rows of logits, probabilities or scores in fp32, bf16 or fp16: how a workgroup or a wavefront walks one in 16-byte pieces wherever it
// begins, and the reductions over it.  All arithmetic is fp32.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ens {

constexpr float LOWEST = -3.402823466e38f;   // running maxima start here: minus infinity less this is minus infinity, not NaN
constexpr float NONE = -__builtin_inff();
constexpr float LOG2E = 1.44269504088896341f;

template <class T> constexpr int PIECE = 16 / (int)sizeof(T);   // elements of 16 bytes

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__bf16 v) { return (float)v; }
__device__ __forceinline__ float up(_Float16 v) { return (float)v; }

__device__ __forceinline__ void unpack(const uint4& u, float (&f)[4], const float*) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(const uint4& u, float (&f)[8], const __bf16*) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; e++) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& u, float (&f)[8], const _Float16*) {
    typedef _Float16 half8 __attribute__((ext_vector_type(8)));
    const half8 h = __builtin_bit_cast(half8, u);
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = (float)h[e];
}
// To the row's type, to nearest even.
__device__ __forceinline__ uint4 pack(const float (&f)[4], const float*) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[8], const __bf16*) {
    typedef float float8 __attribute__((ext_vector_type(8)));
    typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
    const float8 v = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
    return __builtin_bit_cast(uint4, __builtin_convertvector(v, bf8));
}
__device__ __forceinline__ uint4 pack(const float (&f)[8], const _Float16*) {
    typedef float float8 __attribute__((ext_vector_type(8)));
    typedef _Float16 half8 __attribute__((ext_vector_type(8)));
    const float8 v = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
    return __builtin_bit_cast(uint4, __builtin_convertvector(v, half8));
}

// e^((x - m) s) for many x, m their maximum, as one multiply-add and the hardware's power of two (off by one unit): 2^(x c - b) with c = s log2 e
// and b = m c rounded.  The product x c is not rounded, so that a term is off by what c is (2^-24 of the distance x - m, twice) however
// large x is; b's rounding is a factor 2^rest that all terms share: ratios of them need nothing, sums are multiplied by off.  |rest| is 64 at
// most up to a product of 2^31.  Beyond that neighbouring values lie 2^7 / c apart and more, so that no value but m counts whatever c is: a power of
// two makes the product exact and keeps it in range.
struct Exp {
    float c, b, m;
    __device__ __forceinline__ Exp(float max, float s) : m(max) {
        c = s * LOG2E;
        b = m * c;
        if (!(fabsf(b) <= 0x1p31f)) {
            c = __uint_as_float((127u + 40u + 127u - (__float_as_uint(m) >> 23 & 0xFFu)) << 23);   // m c = 2^40 to 2^41
            b = m * c;
        }
    }
    __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_exp2f(fmaf(x, c, -b)); }
    __device__ __forceinline__ float rest() const { return fmaf(m, c, -b); }
    __device__ __forceinline__ float off() const { return __builtin_amdgcn_exp2f(-rest()); }
    // what takes a sum relative to a smaller maximum to this one: parts leave their sums multiplied by off, so that the difference of the maxima is all
    __device__ __forceinline__ float less(float smaller) const { return __builtin_amdgcn_exp2f((smaller - m) * c); }
};

// A whole number in the order of a float that is no NaN, and back.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t key) { return __uint_as_float(key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u)); }

// Over the 64 lanes, the result uniform: shifts within rows of 16 lanes, the rows' last lanes to the next row, lane 31 to the upper half.  Lane 63
// then has them all.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t otherwise) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)otherwise, (int)v, CTRL, ROWS, 0xF, false);
}
template <class V, class F>
__device__ __forceinline__ V lanes_fold(V v, V nothing, F f) {
    static_assert(sizeof(V) == 4, "a register");
    auto with = [&](auto ctrl, auto rows) {
        v = f(v, __builtin_bit_cast(V, moved<decltype(ctrl)::value, decltype(rows)::value>(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, nothing))));
    };
    with(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xF>());    // row_shr 1, 2, 4, 8
    with(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xF>());
    with(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xF>());
    with(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xF>());
    with(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());    // row_bcast 15, 31
    with(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xC>());
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) { return lanes_fold(v, 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; }); }
// (of no NaN: as whole numbers, whose maximum is one instruction a shift where that of floats is four)
__device__ __forceinline__ float lanes_max(float v) { return unordered(lanes_max(ordered(v))); }
__device__ __forceinline__ float lanes_sum(float v) { return lanes_fold(v, 0.f, [](float x, float y) { return x + y; }); }
__device__ __forceinline__ int lanes_sum(int v) { return lanes_fold(v, 0, [](int x, int y) { return x + y; }); }

// A row of `len` elements from `p` on, in any alignment to its elements: the elements in front of a boundary and those behind the last whole
// piece are taken one to a thread, the pieces between them in turn by all.  With 128 threads and more the boundary is a cache line's, so that a
// wavefront's 1 024 bytes are whole lines (rows of odd length otherwise wrote 7 to 19 % more than they hold), with fewer 16 bytes.
template <class T, int THREADS>
struct Row {
    static constexpr int BOUNDARY = THREADS >= 128 ? 128 : 16, HEADS = BOUNDARY / (int)sizeof(T);     // more than elements in front of it
    const T* p;
    int len, head, pieces;
    __device__ __forceinline__ Row(const T* row, int n) : p(row), len(n) {
        head = (int)(-(unsigned)(uintptr_t)row % BOUNDARY) / (int)sizeof(T);
        if (head > n) head = n;
        pieces = (n - head) / PIECE<T>;
    }
    __device__ __forceinline__ const uint4* body() const { return (const uint4*)(p + head); }
    // The single element of this thread, or -1.
    __device__ __forceinline__ int single(int tid) const {
        if (tid < head) return tid;
        const int c = head + pieces * PIECE<T> + tid - HEADS;
        return tid >= HEADS && c < len ? c : -1;
    }
    // f(value, class) over this thread's share
    template <class F>
    __device__ __forceinline__ void each(int tid, F f) const {
        const int one = single(tid);
        if (one >= 0) f(up(p[one]), one);
        for (int i = tid; i < pieces; i += THREADS) {
            float v[PIECE<T>];
            unpack(body()[i], v, p);
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) f(v[e], head + i * PIECE<T> + e);
        }
    }
};

typedef uint32_t Quad __attribute__((ext_vector_type(4)));
// The compiler takes u for a new value from here on: it would keep the unpacked values of a row from one use of it to the next, in twice the registers.
__device__ __forceinline__ void renew(uint4& u) { asm("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w)); }

// This thread's share of a row in registers, PIECES of 16 bytes a thread at most; places behind the row hold minus infinity.  Addresses are
// a scalar for all threads and tid * 16, so that pieces take no address registers each.
template <class T, int THREADS, int PIECES>
struct Held {
    uint4 r[PIECES];
    float one;
    int at;                                                      // class of `one`, or -1
    __device__ __forceinline__ void load(const Row<T, THREADS>& x, int tid) {
        at = x.single(tid);
        const uint32_t mine = (uint32_t)tid * 16u;
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            const char* const at_i = (const char*)(x.body() + i * THREADS);
            if ((i + 1) * THREADS <= x.pieces) r[i] = *(const uint4*)(at_i + mine);
            else {
                r[i] = nothing();
                if (tid < x.pieces - i * THREADS) r[i] = *(const uint4*)(at_i + mine);
            }
        }
        one = at >= 0 ? up(x.p[at]) : NONE;
    }
    // A piece of minus infinity, and a row of it.
    static __device__ __forceinline__ uint4 nothing() {
        const uint32_t none = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __bf16>::value ? 0xFF80FF80u : 0xFC00FC00u;
        return make_uint4(none, none, none, none);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < PIECES; i++) r[i] = nothing();
        one = NONE;
    }
    // f(values of a piece, number of the piece of thread 0) for pieces in reach of the row
    template <class F>
    __device__ __forceinline__ void each(const Row<T, THREADS>& x, F f) {
#pragma unroll
        for (int i = 0; i < PIECES; i++)
            if (i * THREADS < x.pieces) {
                float v[PIECE<T>];
                unpack(r[i], v, x.p);
                f(v, i * THREADS);
                __builtin_amdgcn_sched_barrier(0);               // pieces mixed with each other take registers that hold rows
            }
    }
    __device__ __forceinline__ float max(const Row<T, THREADS>& x) {
        float m = fmaxf(LOWEST, one);
        each(x, [&](const float (&v)[PIECE<T>], int) {
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) m = fmaxf(m, v[e]);
        });
        return m;
    }
    // Minus infinity in the places of marked values: `single` for the single one, a bit each that marks(number of the piece of thread 0) has for a piece's, also
    // for pieces that are not in reach of the row.  The marks of eight pieces are asked for before the first is looked at.
    template <class F>
    __device__ __forceinline__ void hide(const Row<T, THREADS>& x, bool single, F marks) {
        if (single) one = NONE;
#pragma unroll
        for (int first = 0; first < PIECES; first += 8) {
            uint32_t marked[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8 && first + i < PIECES; i++) marked[i / 4] |= marks((first + i) * THREADS) << (i % 4 * 8);
            if (__ballot((marked[0] | marked[1]) != 0) == 0) continue;
#pragma unroll
            for (int i = 0; i < 8 && first + i < PIECES; i++) {
                const uint32_t m = marked[i / 4] >> (i % 4 * 8) & 0xFFu;
                if (__ballot(m != 0) == 0) continue;
                float v[PIECE<T>];
                unpack(r[first + i], v, x.p);
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) v[e] = m >> e & 1 ? NONE : v[e];
                r[first + i] = pack(v, x.p);
            }
        }
    }
    // dst[class] = f(value), dst may be the row
    template <class F>
    __device__ __forceinline__ void map(const Row<T, THREADS>& x, int tid, T* dst, F f) {
        if (at >= 0) dst[at] = (T)f(one);
        const bool alike = (((uintptr_t)dst - (uintptr_t)x.p) & 15u) == 0;
        const uint32_t mine = (uint32_t)tid * 16u;
        each(x, [&](float (&v)[PIECE<T>], int piece) {
            if (tid >= x.pieces - piece) return;
            char* const to = (char*)(dst + x.head + piece * PIECE<T>);
#pragma unroll
            for (int e = 0; e < PIECE<T>; e++) v[e] = f(v[e]);
            if (alike) __builtin_nontemporal_store(__builtin_bit_cast(Quad, pack(v, x.p)), (Quad*)(to + mine));
            else
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) *(T*)(to + mine + e * sizeof(T)) = (T)v[e];
        });
    }
};
// 16 bytes at any multiple of an element: the hardware takes such addresses.  store_past: past the caches, for what is larger than them and for gradients, whose
// rows otherwise push out the rows that are still to be read (4 096 rows of 64 000 fp32 classes with their gradient: 595 us and 398).
typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ uint4 load_loose(const void* p) {
    const Loose v = *(const Loose*)p;
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_loose(void* p, const uint4& u) { *(Loose*)p = Loose{u.x, u.y, u.z, u.w}; }
__device__ __forceinline__ void store_past(void* p, const uint4& u) { __builtin_nontemporal_store(Loose{u.x, u.y, u.z, u.w}, (Loose*)p); }

// N elements (2 to 32 bytes of them) at any multiple of an element.
template <class T, int N>
__device__ __forceinline__ void load_few(const T* p, T (&v)[N]) {
    struct __attribute__((packed, aligned(2))) Few { T v[N]; };
    const Few f = *(const Few*)p;
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = f.v[i];
}
template <class T, int N>
__device__ __forceinline__ void store_few(T* p, const T (&v)[N]) {
    struct __attribute__((packed, aligned(2))) Few { T v[N]; } f;
#pragma unroll
    for (int i = 0; i < N; i++) f.v[i] = v[i];
    *(Few*)p = f;
}

// As Held for a row that is cut where another one is (the row that is written, or for short rows the first one read), wherever it begins itself: classes of
// all rows of a kernel are with the same threads, so that rows of several members can be added in registers.
template <class T, int THREADS, int PIECES>
struct Span {
    uint4 r[PIECES];
    float one;
    // `cut`: the row that sets head, pieces and single
    template <class C>
    __device__ __forceinline__ void load(const T* p, const C& cut, int tid) {
        const uint32_t none = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __bf16>::value ? 0xFF80FF80u : 0xFC00FC00u;
        const uint32_t mine = (uint32_t)tid * 16u;
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            const char* const at = (const char*)(p + cut.head + i * THREADS * PIECE<T>);
            if ((i + 1) * THREADS <= cut.pieces) r[i] = load_loose(at + mine);
            else {
                r[i] = make_uint4(none, none, none, none);
                if (tid < cut.pieces - i * THREADS) r[i] = load_loose(at + mine);
            }
        }
        const int c = cut.single(tid);
        one = c >= 0 ? up(p[c]) : NONE;
    }
    // f(values of piece i, i)
    template <class C, class F>
    __device__ __forceinline__ void each(const C& cut, F f) {
#pragma unroll
        for (int i = 0; i < PIECES; i++)
            if (i * THREADS < cut.pieces) {
                float v[PIECE<T>];
                if (sizeof(T) == 2) renew(r[i]);
                unpack(r[i], v, (const T*)nullptr);
                f(v, i);
                __builtin_amdgcn_sched_barrier(0);
            }
    }
};
// From its start on, without regard to lines.
template <int N>
struct Uncut {
    static constexpr int head = 0;
    int len, pieces;
    __device__ __forceinline__ Uncut(int n) : len(n), pieces(n / N) {}
    __device__ __forceinline__ int single(int tid) const { return pieces * N + tid < len ? pieces * N + tid : -1; }
};
// How a row is cut by what is written: elements of `bytes` each to the next cache line, or to 16 bytes where that may leave more than a wavefront's singles,
// then pieces of N classes.
template <int N, int THREADS>
struct Cut {
    int len, head, pieces, heads;
    __device__ __forceinline__ Cut(const void* to, int bytes, int n) : len(n) {
        const unsigned boundary = THREADS >= 128 || bytes == 4 ? 128 : 16;
        heads = (int)boundary / bytes;
        head = (int)(-(unsigned)(uintptr_t)to % boundary) / bytes;
        if (head > n) head = n;
        pieces = (n - head) / N;
    }
    __device__ __forceinline__ int single(int tid) const {
        if (tid < head) return tid;
        const int c = head + pieces * N + tid - heads;
        return tid >= heads && c < len ? c : -1;
    }
};
// Stores PIECE<T> floats of a row, `to` at any multiple of 4 bytes.
template <int N>
__device__ __forceinline__ void store_floats(float* to, const float (&v)[N], bool past) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const uint4 u = make_uint4(__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3]));
        if (past) store_past(to + e, u);
        else store_loose(to + e, u);
    }
}
template <int N>
__device__ __forceinline__ void load_floats(const float* from, float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const uint4 u = load_loose(from + e);
        v[e] = __uint_as_float(u.x); v[e + 1] = __uint_as_float(u.y); v[e + 2] = __uint_as_float(u.z); v[e + 3] = __uint_as_float(u.w);
    }
}

template <int N>
__device__ __forceinline__ float sum_of(const float (&v)[N]) {
    if constexpr (N == 8) return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    else return (v[0] + v[1]) + (v[2] + v[3]);
}

// Between the wavefronts of a workgroup, or the lanes of the only one.
template <int THREADS>
__device__ __forceinline__ void group_sync() {
    if constexpr (THREADS > 64) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Over a workgroup; `box`: a float for each of its wavefronts.  Every thread gets the result, added or compared in the same order.
template <int THREADS>
__device__ __forceinline__ float group_max(float v, float* box) {
    v = lanes_max(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
        __syncthreads();
        v = box[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; w++) v = fmaxf(v, box[w]);
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float v, float* box) {
    v = lanes_sum(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
        __syncthreads();
        v = box[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; w++) v += box[w];
    }
    return v;
}

// Calls f with a value of the type that `dtype` (ENS_FP32, ENS_BF16, ENS_FP16) names.
template <class F>
static inline hipError_t by_type(int dtype, F f) {
    switch (dtype) {
        case 0: return f((float)0);
        case 1: return f((__bf16)0.f);
        case 2: return f((_Float16)0.f);
    }
    return hipErrorInvalidValue;
}

}  // namespace ens
