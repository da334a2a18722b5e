// The k best classes of a row, the lowest class first among equal values, NaN below everything.
//
// A workgroup (a wavefront for short rows) holds the row in registers.  Of the maxima of 64 to 256 groups of its lanes the k-th largest, t, is a
// bound: k values at least are no smaller.  What is not smaller (some k (1 + k / groups) values where the row is in no order) is collected in
// LDS and ranked by comparing every pair, as 64-bit keys: 32 bits in the order of the values, then the class.  Everything is one look at the row for
// the maxima, a second one at the pieces that hold something, and a third for the sum of a softmax.
// Where too many values are no smaller than t (equal ones, most of the row masked, the large ones in few lanes), or too few (NaN), the bound is found
// by halving, over the row in memory.
// Rows that are longer than that go in parts, each part's best to the workspace, and a second launch chooses among them.
// Bound by memory where k is small: 1 500 rows of 50 001 16-bit classes for k = 5 take 31 us (4.8 TB/s).  The softmax's powers add 6 us to them, k = 100 10 more:
// comparing the 256 maxima, reading some 130 pieces again, ranking as many keys, while the compute unit's other row loads (47 us with both).
// 8 100 rows of 1 000 fp32 classes, k = 5: 11.3 us, 2.9 TB/s.  One row of 128 000: 12.5 us.  In parts, k = 50: one row of 300 000 18 us, 40 of them 21.
// With 4 pieces a thread and a wavefront to four, 2 to 23 of 80 registers are spilled (most in 16 bits and four wavefronts).
#include <algorithm>

#include "operators.h"
#include "rows.h"

namespace ens {

enum { TOP_VALUE = 0, TOP_LOG = 1, TOP_LOG_SOFTMAX = 2 };
constexpr int TOP_ROOM = 1024, TOP_WAVE_ROOM = 256;     // candidates in LDS
constexpr int TOP_WAVE_K = 48, TOP_PAIR_K = 96;         // for which 64 and 128 groups, the lanes of one and two wavefronts, are enough
constexpr int JOIN_THREADS = 1024, JOIN_KEYS = 2048;    // keys of a row's parts: 8 for each of 256 groups, so that those of 128 groups have room

__device__ __forceinline__ uint32_t key_of(float v) { return v != v ? 0u : ordered(v + 0.f); }      // both zeros are one
__device__ __forceinline__ float value_of(uint32_t key) { return key == 0u ? __uint_as_float(0x7FC00000u) : unordered(key); }
// Larger value first, then lower class; no key is 0.
__device__ __forceinline__ uint64_t key_of(float v, int c) { return (uint64_t)key_of(v) << 32 | (0xFFFFFFFFu - (uint32_t)c); }

// What is written of a value.  Halves: the difference of two fp32 values may not be one, where it is one at the temperature.
template <bool LSE>
__device__ __forceinline__ float answer(const TopArgs& a, float v, float mx, float shift) {
    if constexpr (LSE) return (0.5f * v - 0.5f * mx) * a.inv_temperature * 2.f - shift;
    return a.form == TOP_LOG ? logf(v) : v;
}

template <int THREADS>
__device__ __forceinline__ int group_count(int v, float* box) {
    v = lanes_sum(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = __int_as_float(v);
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; w++) v += __float_as_int(box[w]);
    }
    return v;
}

// The best k of a row that holds k values at least, by halving the interval of keys that the k-th lies in: into found[0 .. ), k of them at least and
// `room` at most.  Returns how many.
template <class T, int THREADS>
__device__ __attribute__((noinline)) int halve(const T* p, int len, int base, int k, int room, uint64_t* found, int* count, float* box) {
    const int tid = threadIdx.x;
    const Row<T, THREADS> x(p, len);
    auto larger = [&](uint32_t than) {
        int c = 0;
        x.each(tid, [&](float v, int) { c += key_of(v) > than; });
        return group_count<THREADS>(c, box);
    };
    // k values at least are not smaller than t, fewer than k are larger than high
    uint32_t t = 0, high = 0xFFFFFFFFu;
    int above = larger(t);
    if (above >= k && above > room) {
        while (high - t > 1u) {
            const uint32_t middle = t + (high - t) / 2;
            const int c = larger(middle);
            if (c >= k) t = middle, above = c;
            else high = middle;
            if (c >= k && c <= room) break;
        }
        if (above > room) {                                      // the k-th value is `high` itself
            t = high;
            above = larger(t);
        }
    }
    group_sync<THREADS>();
    if (tid == 0) *count = 0;
    group_sync<THREADS>();
    x.each(tid, [&](float v, int c) {
        const uint32_t key = key_of(v);
        if (key > t) found[atomicAdd(count, 1)] = (uint64_t)key << 32 | (0xFFFFFFFFu - (uint32_t)(base + c));
    });
    group_sync<THREADS>();
    int have = above;
    // and the lowest of those that equal t, in order
    for (int c0 = 0; have < k && c0 < len; c0 += THREADS) {
        const int c = c0 + tid;
        const bool hit = c < len && key_of(up(p[c])) == t;
        const unsigned long long mask = __ballot(hit);
        int at = have + __popcll(mask & ((1ull << (tid & 63)) - 1));
        if constexpr (THREADS > 64) {
            __syncthreads();
            if ((tid & 63) == 0) box[tid >> 6] = __int_as_float(__popcll(mask));
            __syncthreads();
            for (int w = 0; w < THREADS / 64; w++) {
                if (w < tid >> 6) at += __float_as_int(box[w]);
                have += __float_as_int(box[w]);
            }
        } else have += __popcll(mask);
        if (hit && at < k) found[at] = (uint64_t)t << 32 | (0xFFFFFFFFu - (uint32_t)(base + c));
    }
    group_sync<THREADS>();
    return above < k ? k : above;
}

// Calls f(rank, key) for the best k of `have` different keys in LDS, in no order.  Up to eight threads share a key's comparisons, and read sixteen keys
// ahead of them, which would otherwise wait for each; there is room for zeros behind the last key.
constexpr int AHEAD = 16;
template <int THREADS, class F>
__device__ __forceinline__ void rank_keys(uint64_t* found, int have, int k, F f) {
    const int padded = (have + AHEAD - 1) / AHEAD * AHEAD, tid = threadIdx.x;
    if (tid < padded - have) found[have + tid] = 0;
    group_sync<THREADS>();
    int share = 1;
    if constexpr (THREADS > 64)
        while (share < 8 && 2 * share * have <= THREADS) share *= 2;
    for (int first = 0; first < have; first += THREADS / share) {
        const int i = first + tid / share;
        const uint64_t one = i < have ? found[i] : 0;
        int at = 0;
        for (int o = tid % share * AHEAD; o < padded; o += share * AHEAD) {
            uint64_t other[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; e++) other[e] = found[o + e];
#pragma unroll
            for (int e = 0; e < AHEAD; e++) at += other[e] > one;
        }
        if constexpr (THREADS > 64)
            for (int o = 1; o < share; o *= 2) at += __shfl_xor(at, o, 64);
        if (i < have && tid % share == 0 && at < k) f(at, one);
    }
}

struct TopParts {
    int parts, length;                                           // classes of every part but the last
    // of the workspace, in 8 bytes: k keys for each part of each row, then a maximum and a sum for each
    __host__ __device__ int64_t keys(int64_t n, int k) const { return n * parts * k; }
    __host__ __device__ int64_t bytes(int64_t n, int k) const { return parts == 1 ? 0 : 8 * (keys(n, k) + n * parts); }
};

// The k-th largest of the maxima of `groups` groups of lanes, as a bound (t): `own` is the largest of this thread's values.  A group is up to eight
// neighbouring lanes, which share its comparisons.  *bound is 0 before.  LSE: also the row's maximum and its sum of powers, of which powers(Exp) is
// this thread's share, between the same two barriers.
struct Bound { float t, mx, sum; };
template <int THREADS, bool LSE, class F>
__device__ __forceinline__ Bound find_bound(float own, int groups, int k, float scale, float* maxima, uint32_t* bound, float* box, F powers) {
    const int tid = threadIdx.x, lane = tid & 63, member = THREADS / groups, some = groups / member;
    float folded = own;
    for (int o = 1; o < member; o <<= 1) folded = fmaxf(folded, __shfl_xor(folded, o, 64));
    if (tid % member == 0) maxima[tid / member] = folded;
    group_sync<THREADS>();
    const float* const theirs = maxima + tid % member * some;
    int no_smaller = 0;
    for (int i = 0; i < some; i += AHEAD / 2) {
        float4 m[AHEAD / 8];
#pragma unroll
        for (int e = 0; e < AHEAD / 8; e++) m[e] = *(const float4*)&theirs[i + 4 * e];
#pragma unroll
        for (int e = 0; e < AHEAD / 8; e++) no_smaller += (m[e].x >= folded) + (m[e].y >= folded) + (m[e].z >= folded) + (m[e].w >= folded);
    }
    for (int o = 1; o < member; o <<= 1) no_smaller += __shfl_xor(no_smaller, o, 64);
    const float reached = lanes_max(no_smaller >= k ? folded : LOWEST);      // the largest that k of them reach
    if (lane == 0) atomicMax(bound, key_of(reached));
    Bound found{0.f, LOWEST, 0.f};
    float off = 1.f;
    if (LSE) {
        for (int i = lane; i < groups; i += 64) found.mx = fmaxf(found.mx, maxima[i]);
        found.mx = lanes_max(found.mx);
        const Exp power(found.mx, scale);
        off = power.off();
        found.sum = lanes_sum(powers(power));
        if (lane == 0) box[tid >> 6] = found.sum;
    }
    group_sync<THREADS>();
    if (LSE) {
        found.sum = box[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; w++) found.sum += box[w];
        found.sum *= off;
    }
    found.t = value_of(*bound);
    return found;
}

// Short rows for many of their values: fewer pieces of 16 bytes than twice k.  The values are dealt to the threads one by one, so that each has one of the
// row's parts; otherwise as below.
template <class T, int THREADS, int EACH, bool LSE>
__global__ __launch_bounds__(THREADS) void top_dealt_kernel(const TopArgs a) {
    constexpr int ROOM = THREADS == 64 ? TOP_WAVE_ROOM : TOP_ROOM;
    __shared__ __align__(16) uint64_t found[ROOM + AHEAD];
    __shared__ __align__(16) float maxima[THREADS];
    __shared__ float box[16];
    __shared__ uint32_t bound;
    __shared__ int count;
    const int tid = threadIdx.x, k = a.k;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.values + row * a.ld;
        float v[EACH], own = LOWEST;
#pragma unroll
        for (int i = 0; i < EACH; i++) v[i] = tid + i * THREADS < a.classes ? up(p[tid + i * THREADS]) : NONE;
#pragma unroll
        for (int i = 0; i < EACH; i++) own = fmaxf(own, v[i]);
        if (tid == 0) {
            bound = 0;
            count = 0;
        }
        const Bound top = find_bound<THREADS, LSE>(own, THREADS, k, a.inv_temperature, maxima, &bound, box, [&](const Exp& power) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < EACH; i++) sum += power(v[i]);
            return sum;
        });
        const float t = top.t, mx = top.mx, sum = top.sum;
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (v[i] >= t && tid + i * THREADS < a.classes) {
                const int at = atomicAdd(&count, 1);
                if (at < ROOM) found[at] = key_of(v[i], tid + i * THREADS);
            }
        group_sync<THREADS>();
        int have = count;
        if (have > ROOM || have < k) have = halve<T, THREADS>(p, a.classes, 0, k, ROOM, found, &count, box);
        const float shift = LSE ? sum == 0.f ? 0.f : logf(sum) : 0.f;
        rank_keys<THREADS>(found, have, k, [&](int at, uint64_t key) {
            const float x = value_of((uint32_t)(key >> 32));
            a.index[row * k + at] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
            a.value[row * k + at] = answer<LSE>(a, x, mx, shift);
        });
        group_sync<THREADS>();
    }
}

template <class T, int THREADS, int PIECES, bool LSE>
__global__ __launch_bounds__(THREADS, PIECES == 16 ? 4 : 6) void top_held_kernel(const TopArgs a, const TopParts split) {
    constexpr int ROOM = THREADS == 64 ? TOP_WAVE_ROOM : TOP_ROOM, MOST = THREADS < 256 ? THREADS : 256;
    constexpr bool AGAIN = PIECES > 4;
    __shared__ __align__(16) uint64_t found[ROOM + AHEAD];
    __shared__ __align__(16) float maxima[MOST];
    __shared__ float box[16];
    __shared__ uint32_t bound;
    __shared__ int count, listed;
    __shared__ uint16_t pieces[AGAIN ? ROOM : 1];
    const int tid = threadIdx.x, k = a.k;
    for (int64_t job = blockIdx.x; job < a.n * split.parts; job += gridDim.x) {
        const int64_t row = split.parts == 1 ? job : job / split.parts;
        const int part = (int)(job - row * split.parts), first = part * split.length, length = min(split.length, a.classes - first);
        const T* const p = (const T*)a.values + row * a.ld + first;
        const Row<T, THREADS> x(p, length);
        // more than k, so that few values exceed the bound, but with many comparisons of their own (at k = 85 of 128 groups 36 us against 39 of 256, at k = 110
        // 51 against 43: 3 000 rows of 20 000 fp16); as many as there are where not all threads have a piece; eight lanes of a group at most
        const int groups = THREADS == 64 ? 64 : x.pieces < THREADS ? MOST : min(MOST, max(k <= 32 ? 64 : k <= TOP_PAIR_K ? 128 : 256, THREADS / 8));
        Held<T, THREADS, PIECES> held;
        held.load(x, tid);
        float own = fmaxf(LOWEST, held.one), most[PIECES];       // LOWEST for nothing but minus infinity
#pragma unroll
        for (int i = 0; i < PIECES; i++) most[i] = NONE;
        held.each(x, [&](const float (&v)[PIECE<T>], int piece) {
            float m = v[0];
#pragma unroll
            for (int e = 1; e < PIECE<T>; e++) m = fmaxf(m, v[e]);
            if (AGAIN) most[piece / THREADS] = m;
            own = fmaxf(own, m);
        });
        if (tid == 0) {
            bound = 0;
            count = 0;
            listed = 0;
        }
        const Bound top = find_bound<THREADS, LSE>(own, groups, k, a.inv_temperature, maxima, &bound, box, [&](const Exp& power) {
            float sum = power(held.one);
            held.each(x, [&](const float (&v)[PIECE<T>], int) {
                float e[PIECE<T>];
#pragma unroll
                for (int i = 0; i < PIECE<T>; i++) e[i] = power(v[i]);
                sum += sum_of(e);
            });
            return sum;
        });
        const float t = top.t, mx = top.mx, sum = top.sum;
        auto take = [&](float v, int c) {
            if (!(v >= t)) return;
            const int at = atomicAdd(&count, 1);
            if (at < ROOM) found[at] = key_of(v, first + c);
        };
        if (held.at >= 0) take(held.one, held.at);
        if constexpr (AGAIN) {
            // some k pieces hold one: listed, and read again from the cache, a thread a value (all pieces of their threads would be nearly all of the row's lines)
            uint32_t hits = 0;
#pragma unroll
            for (int i = 0; i < PIECES; i++) hits |= most[i] >= t ? 1u << i : 0u;
            if (hits) {
                int at = atomicAdd(&listed, __popc(hits));
                for (; hits; hits &= hits - 1, at++)
                    if (at < ROOM) pieces[at] = (uint16_t)((__ffs(hits) - 1) * THREADS + tid);
                    else count = ROOM + 1;                       // more than ROOM values then
            }
            __syncthreads();
            for (int i = tid; i < min(listed, ROOM) * PIECE<T>; i += THREADS) {
                const int c = x.head + pieces[i / PIECE<T>] * PIECE<T> + i % PIECE<T>;
                take(up(p[c]), c);
            }
        } else {
            held.each(x, [&](const float (&v)[PIECE<T>], int piece) {
                float m = v[0];
#pragma unroll
                for (int e = 1; e < PIECE<T>; e++) m = fmaxf(m, v[e]);
                if (!(m >= t) || tid >= x.pieces - piece) return;
#pragma unroll
                for (int e = 0; e < PIECE<T>; e++) take(v[e], x.head + (piece + tid) * PIECE<T> + e);
            });
        }
        group_sync<THREADS>();
        int have = count;
        const int want = min(k, length);
        if (have > ROOM || have < want) have = halve<T, THREADS>(p, length, first, want, ROOM, found, &count, box);
        if (split.parts == 1) {
            const float shift = LSE ? sum == 0.f ? 0.f : logf(sum) : 0.f;      // a row of minus infinities keeps them
            rank_keys<THREADS>(found, have, k, [&](int at, uint64_t key) {
                const float v = value_of((uint32_t)(key >> 32));
                a.index[row * k + at] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
                a.value[row * k + at] = answer<LSE>(a, v, mx, shift);
            });
        } else {
            uint64_t* const out = (uint64_t*)a.workspace + job * k;
            rank_keys<THREADS>(found, have, want, [&](int at, uint64_t key) { out[at] = key; });
            for (int i = want + tid; i < k; i += THREADS) out[i] = 0;
            if (tid == 0) ((float2*)a.workspace)[split.keys(a.n, k) + job] = make_float2(mx, sum);
        }
        group_sync<THREADS>();
    }
}

// Among the keys that the parts of a row left.  They are dealt to groups of four threads in turn, so that a part's best are with as many groups; k of
// the groups' maxima reach the k-th largest of them, and what those groups hold has room.
template <bool LSE>
__global__ __launch_bounds__(JOIN_THREADS) void top_join_kernel(const TopArgs a, const TopParts split) {
    constexpr int EACH = JOIN_KEYS / JOIN_THREADS, GROUPS = 256, MEMBER = JOIN_THREADS / GROUPS;
    __shared__ __align__(16) uint64_t found[JOIN_KEYS / GROUPS * TOP_MAX_K + AHEAD], maxima[GROUPS];
    __shared__ uint64_t bound;
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, k = a.k;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const uint64_t* const in = (const uint64_t*)a.workspace + row * split.parts * k;
        uint64_t mine[EACH], best = 0;
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int at = (i * MEMBER + tid % MEMBER) * GROUPS + tid / MEMBER;
            mine[i] = at < split.parts * k ? in[at] : 0;
            best = mine[i] > best ? mine[i] : best;
        }
        float mx = LOWEST, sum = 0.f;
        if (LSE) {                                               // every wavefront for itself
            const float2* const from = (const float2*)a.workspace + split.keys(a.n, k) + row * split.parts;
            for (int i = lane; i < split.parts; i += 64) mx = fmaxf(mx, from[i].x);
            mx = lanes_max(mx);
            const Exp power(mx, a.inv_temperature);
            for (int i = lane; i < split.parts; i += 64) sum += from[i].y * power.less(from[i].x);
            sum = lanes_sum(sum);
        }
#pragma unroll
        for (int o = 1; o < MEMBER; o *= 2) {
            const uint64_t other = __shfl_xor(best, o, 64);
            best = other > best ? other : best;
        }
        if (tid % MEMBER == 0) maxima[tid / MEMBER] = best;
        if (tid == 0) {
            count = 0;
            bound = 0;
        }
        __syncthreads();
        int larger = 0;
#pragma unroll
        for (int i = 0; i < GROUPS / MEMBER; i += AHEAD) {
            uint64_t other[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; e++) other[e] = maxima[tid % MEMBER * (GROUPS / MEMBER) + i + e];
#pragma unroll
            for (int e = 0; e < AHEAD; e++) larger += other[e] > best;
        }
#pragma unroll
        for (int o = 1; o < MEMBER; o *= 2) larger += __shfl_xor(larger, o, 64);
        if (larger == k - 1 && best && tid % MEMBER == 0) bound = best;      // (fewer than k groups with keys: all keys)
        __syncthreads();
        const uint64_t t = bound ? bound : 1;
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (mine[i] >= t) found[atomicAdd(&count, 1)] = mine[i];
        __syncthreads();
        const float shift = LSE ? sum == 0.f ? 0.f : logf(sum) : 0.f;
        rank_keys<JOIN_THREADS>(found, count, k, [&](int at, uint64_t key) {
            const float v = value_of((uint32_t)(key >> 32));
            a.index[row * k + at] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
            a.value[row * k + at] = answer<LSE>(a, v, mx, shift);
        });
        __syncthreads();
    }
}

// Rows that are too long for the keys of their parts: a workgroup walks each in memory.
template <class T, bool LSE>
__global__ __launch_bounds__(1024) void top_long_kernel(const TopArgs a) {
    __shared__ __align__(16) uint64_t found[TOP_ROOM + AHEAD];
    __shared__ float box[16];
    __shared__ int count;
    const int tid = threadIdx.x, k = a.k;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* const p = (const T*)a.values + row * a.ld;
        float mx = LOWEST, shift = 0.f;
        if (LSE) {
            const Row<T, 1024> x(p, a.classes);
            x.each(tid, [&](float v, int) { mx = fmaxf(mx, v); });
            mx = group_max<1024>(mx, box);
            const Exp power(mx, a.inv_temperature);
            float sum = 0.f;
            x.each(tid, [&](float v, int) { sum += power(v); });
            sum = group_sum<1024>(sum, box);
            shift = sum == 0.f ? 0.f : logf(sum * power.off());
        }
        const int have = halve<T, 1024>(p, a.classes, 0, k, TOP_ROOM, found, &count, box);
        rank_keys<1024>(found, have, k, [&](int at, uint64_t key) {
            const float v = value_of((uint32_t)(key >> 32));
            a.index[row * k + at] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
            a.value[row * k + at] = answer<LSE>(a, v, mx, shift);
        });
        __syncthreads();
    }
}

// How rows are cut; parts 0: too long.  A row that a workgroup's registers hold stays whole, also where there is only one: 128 000 bf16 classes take
// 12.3 us whole, as a call from Python, and 16 in 32 parts with the second launch; 32 000 take 11.3 and 15.3, and of 64 and 200 rows 11.3 to
// 20 and 18 to 31.
static TopParts split_top(int classes, int k, int dtype) {
    const int pieces = classes / (dtype == 0 ? 4 : 8), parts = pieces > 16384 ? (pieces + 8191) / 8192 : 1;
    if (parts > std::max(1, JOIN_KEYS / k)) return TopParts{0, 0};
    const int length = ((classes + parts - 1) / parts + 63) / 64 * 64;
    return TopParts{(classes + length - 1) / length, length};
}

int64_t top_workspace(int64_t n, int classes, int k, int dtype) {
    const TopParts split = split_top(classes, k, dtype);
    return split.parts ? split.bytes(n, k) : 0;
}

template <class T, int THREADS, int PIECES>
static void launch_top_held(const TopArgs& a, const TopParts& split, hipStream_t s) {
    const dim3 grid((unsigned)std::min<int64_t>(a.n * split.parts, 1 << 14)), group(THREADS);
    if (a.form == TOP_LOG_SOFTMAX) hipLaunchKernelGGL((top_held_kernel<T, THREADS, PIECES, true>), grid, group, 0, s, a, split);
    else hipLaunchKernelGGL((top_held_kernel<T, THREADS, PIECES, false>), grid, group, 0, s, a, split);
}

template <class T, int THREADS>
static void launch_top_dealt(const TopArgs& a, hipStream_t s) {
    const dim3 rows((unsigned)std::min<int64_t>(a.n, 1 << 14)), group(THREADS);
    if (a.form == TOP_LOG_SOFTMAX) hipLaunchKernelGGL((top_dealt_kernel<T, THREADS, 8, true>), rows, group, 0, s, a);
    else hipLaunchKernelGGL((top_dealt_kernel<T, THREADS, 8, false>), rows, group, 0, s, a);
}

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    const TopParts split = split_top(a.classes, a.k, a.dtype);
    return by_type(a.dtype, [&](auto t) {
        typedef decltype(t) T;
        const dim3 rows((unsigned)std::min<int64_t>(a.n, 1 << 14));
        if (split.parts == 0) {
            if (a.form == TOP_LOG_SOFTMAX) hipLaunchKernelGGL((top_long_kernel<T, true>), rows, dim3(1024), 0, s, a);
            else hipLaunchKernelGGL((top_long_kernel<T, false>), rows, dim3(1024), 0, s, a);
            return hipGetLastError();
        }
        const int pieces = split.length / PIECE<T>;
        // a wavefront or two take a short row where their lanes are groups enough: 8 100 rows of 1 000 classes for k = 50 took 53 to 60 us with four
        if (pieces < 2 * a.k && a.classes <= 256 * 8) {
            if (a.classes <= 64 * 8 && a.k <= TOP_WAVE_K) launch_top_dealt<T, 64>(a, s);
            else if (a.classes <= 128 * 8 && a.k <= TOP_PAIR_K) launch_top_dealt<T, 128>(a, s);
            else launch_top_dealt<T, 256>(a, s);
            return hipGetLastError();
        }
        if (pieces <= 64 * 4 && a.k <= TOP_WAVE_K) launch_top_held<T, 64, 4>(a, split, s);
        else if (pieces <= 128 * 4 && a.k <= TOP_PAIR_K) launch_top_held<T, 128, 4>(a, split, s);
        else if (pieces <= 256 * 4) launch_top_held<T, 256, 4>(a, split, s);
        else if (pieces <= 256 * 16) launch_top_held<T, 256, 16>(a, split, s);
        else if (pieces <= 512 * 16) launch_top_held<T, 512, 16>(a, split, s);
        else launch_top_held<T, 1024, 16>(a, split, s);
        if (split.parts > 1) {
            if (a.form == TOP_LOG_SOFTMAX) hipLaunchKernelGGL((top_join_kernel<true>), rows, dim3(JOIN_THREADS), 0, s, a, split);
            else hipLaunchKernelGGL((top_join_kernel<false>), rows, dim3(JOIN_THREADS), 0, s, a, split);
        }
        return hipGetLastError();
    });
}

}  // namespace ens
