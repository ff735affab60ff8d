// Log probabilities of given tokens over [T, V] logits, with each row's entropy and most likely alternatives, and their gradient with
// respect to the logits.  Per row, with c the inverse temperature, m = max z and d_j = c (z_j - m) <= 0:
//     s = sum exp d_j,    log p_j = d_j - log s,    H = log s - (sum exp(d_j) d_j) / s
// in one pass over the row: every thread keeps its own maximum and sums relative to it and corrects them when the maximum moves.
#include "common.cuh"
#include "device_state.h"
#include "f32x2.cuh"
#include "launch.h"

namespace qlora {

constexpr int LP_BWD_THREADS = 512;
constexpr int LP_UNROLL = 4;             // 16-byte vectors that a thread has on their way at a time
constexpr int LP_CLUSTER = 8;            // most blocks that share a row
constexpr int LP_GROUPS = 128;           // most groups of threads whose maxima bound the alternatives
constexpr int LP_CANDIDATES = 512;       // entries that are put in order together
static_assert(LP_CANDIDATES >= LP_CLUSTER * QLORA_MAX_TOP, "the lists of a cluster are merged in the same place");
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float lp_f(float x) { return x; }
__device__ __forceinline__ float lp_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float lp_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T lp_to(float x);
template <> __device__ __forceinline__ float lp_to<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 lp_to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half lp_to<__half>(float x) { return __float2half_rn(x); }

// The larger of two, NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 16 bytes of a row as pairs of fp32, and their maximum in the form they lie in memory.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ f2 pair(const uint4& v, int i) { return i == 0 ? make_f2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_f2(__uint_as_float(v.z), __uint_as_float(v.w)); }
    typedef float Max;
    static __device__ __forceinline__ Max lowest() { return -INFINITY; }
    static __device__ __forceinline__ Max fold(Max m, const uint4& v) {
        return max_nan(max_nan(m, max_nan(__uint_as_float(v.x), __uint_as_float(v.y))), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float value(Max m) { return m; }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    static __device__ __forceinline__ f2 pair(const uint4& v, int i) { return unpack_bf16(word(v, i)); }
    typedef __nv_bfloat162 Max;
    static __device__ __forceinline__ Max lowest() { return __float2bfloat162_rn(-INFINITY); }
    static __device__ __forceinline__ Max of(uint32_t w) { return *reinterpret_cast<const Max*>(&w); }
    static __device__ __forceinline__ Max fold(Max m, const uint4& v) {
        return __hmax2_nan(__hmax2_nan(m, __hmax2_nan(of(v.x), of(v.y))), __hmax2_nan(of(v.z), of(v.w)));
    }
    static __device__ __forceinline__ float value(Max m) { return max_nan(__low2float(m), __high2float(m)); }
};
template <> struct Vec<__half> {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    static __device__ __forceinline__ f2 pair(const uint4& v, int i) {
        const uint32_t w = word(v, i);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return make_f2(f.x, f.y);
    }
    typedef __half2 Max;
    static __device__ __forceinline__ Max lowest() { return __float2half2_rn(-INFINITY); }
    static __device__ __forceinline__ Max of(uint32_t w) { return *reinterpret_cast<const Max*>(&w); }
    static __device__ __forceinline__ Max fold(Max m, const uint4& v) {
        return __hmax2_nan(__hmax2_nan(m, __hmax2_nan(of(v.x), of(v.y))), __hmax2_nan(of(v.z), of(v.w)));
    }
    static __device__ __forceinline__ float value(Max m) { return max_nan(__low2float(m), __high2float(m)); }
};

// A row of V elements that begins anywhere: `head` elements up to the first 16-byte boundary, whole vectors, the rest.
template <typename T>
struct RowParts {
    const T* z;
    int head, vectors, tail, rest;       // tail: where the last `rest` elements begin
    __device__ __forceinline__ RowParts(const T* row, int V) : z(row) {
        head = min(V, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(row)) & 15u) / (int)sizeof(T));
        vectors = (V - head) / Vec<T>::N;
        tail = head + vectors * Vec<T>::N;
        rest = V - tail;
    }
    __device__ __forceinline__ const uint4* body() const { return reinterpret_cast<const uint4*>(z + head); }
};

__device__ __forceinline__ uint4 load_stream(const uint4* p) {          // read once, not kept in L1
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// The order of the alternatives: larger logits first (a NaN before all, -0 with 0), equal ones by their place.  Larger keys come first.
__device__ __forceinline__ uint32_t order_key(float z) {
    if (z != z) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t entry_key(uint32_t key, int j) { return (uint64_t)key << 32 | (uint32_t)~j; }
__device__ __forceinline__ int entry_place(uint64_t e) { return (int)~(uint32_t)e; }
__device__ __forceinline__ float entry_logit(uint64_t e) {
    const uint32_t key = (uint32_t)(e >> 32);
    return key == 0xFFFFFFFFu ? __int_as_float(0x7FC00000) : __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// A maximum and sums relative to it: s = sum exp(c (z - m)), a = sum exp(c (z - m)) (z - m).  kd = c log2(e).
struct RowSums {
    float m, s, a;
};
// Moves the sums to a maximum m >= x.m.  (Nothing yet, or a row without a distribution: the factor is 0 or NaN, the sums become 0.)
__device__ __forceinline__ void rebase(RowSums& x, float m, float kd) {
    const float d = x.m - m, e = fast_exp2(d * kd);
    x.a = e > 0.f ? e * fmaf(x.s, d, x.a) : 0.f;
    x.s = e > 0.f ? x.s * e : 0.f;
    x.m = m;
}
// Adds a pair of logits at most x.m.  A masked one is -inf, or x.m is: the difference becomes the lowest number, its exponential 0, and
// their product 0 instead of NaN.
__device__ __forceinline__ void add_pair(f2& s2, f2& a2, f2 z, f2 minus_m, f2 kd2) {
    const f2 raw = add2(z, minus_m);
    const f2 d = make_f2(fmaxf(lo_of(raw), -3.0e38f), fmaxf(hi_of(raw), -3.0e38f));
    const f2 e = exp2_2(mul2(d, kd2));
    s2 = add2(s2, e);
    a2 = fma2(e, d, a2);
}
__device__ __forceinline__ void add_one(RowSums& x, float z, float kd) {
    const float m = max_nan(x.m, z);
    if (m != x.m) rebase(x, m, kd);
    const float d = fmaxf(z - m, -3.0e38f), e = fast_exp2(d * kd);
    x.s += e;
    x.a = fmaf(e, d, x.a);
}
// Sums of a warp's lanes, the same in all of them.
__device__ __forceinline__ RowSums warp_merge(RowSums x, float kd) {
    float m = x.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    rebase(x, m, kd);
    return RowSums{m, warp_sum(x.s), warp_sum(x.a)};
}

// The sums of this thread's part of the row.
template <typename T, int THREADS>
__device__ __forceinline__ RowSums thread_sums(const RowParts<T>& row, float kd) {
    RowSums x{-INFINITY, 0.f, 0.f};
    const f2 kd2 = make_f2(kd, kd);
    const uint4* body = row.body();
    for (int c0 = threadIdx.x; c0 < row.vectors; c0 += LP_UNROLL * THREADS) {
        uint4 v[LP_UNROLL];
        typename Vec<T>::Max top = Vec<T>::lowest();
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * THREADS < row.vectors) v[u] = load_stream(body + c0 + u * THREADS);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * THREADS < row.vectors) top = Vec<T>::fold(top, v[u]);
        const float m = max_nan(x.m, Vec<T>::value(top));
        if (m != x.m) rebase(x, m, kd);
        const f2 minus_m = make_f2(-m, -m);
        f2 s2 = make_f2(x.s, 0.f), a2 = make_f2(x.a, 0.f);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * THREADS < row.vectors) {
#pragma unroll
                for (int i = 0; i < Vec<T>::N / 2; ++i) add_pair(s2, a2, Vec<T>::pair(v[u], i), minus_m, kd2);
            }
        x.s = lo_of(s2) + hi_of(s2);
        x.a = lo_of(a2) + hi_of(a2);
    }
    if ((int)threadIdx.x < row.head) add_one(x, lp_f(row.z[threadIdx.x]), kd);
    if ((int)threadIdx.x < row.rest) add_one(x, lp_f(row.z[row.tail + threadIdx.x]), kd);
    return x;
}

// Calls f(key, place) for this thread's logits of the part of the row (the same ones as in thread_sums) whose key is at least `least`.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void each_from(const RowParts<T>& row, uint32_t least, F f) {
    const uint4* body = row.body();
    for (int c0 = threadIdx.x; c0 < row.vectors; c0 += LP_UNROLL * THREADS) {
        uint4 v[LP_UNROLL];
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * THREADS < row.vectors) v[u] = body[c0 + u * THREADS];
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) {
            if (c0 + u * THREADS >= row.vectors || order_key(Vec<T>::value(Vec<T>::fold(Vec<T>::lowest(), v[u]))) < least) continue;
#pragma unroll
            for (int i = 0; i < Vec<T>::N; ++i) {
                const f2 pr = Vec<T>::pair(v[u], i / 2);
                const uint32_t key = order_key(i & 1 ? hi_of(pr) : lo_of(pr));
                if (key >= least) f(key, row.head + (c0 + u * THREADS) * Vec<T>::N + i);
            }
        }
    }
    if ((int)threadIdx.x < row.head) {
        const uint32_t key = order_key(lp_f(row.z[threadIdx.x]));
        if (key >= least) f(key, (int)threadIdx.x);
    }
    if ((int)threadIdx.x < row.rest) {
        const uint32_t key = order_key(lp_f(row.z[row.tail + threadIdx.x]));
        if (key >= least) f(key, row.tail + (int)threadIdx.x);
    }
}

struct TopShared {
    uint64_t cand[LP_CANDIDATES];        // entries that may be among the largest; in the first block of a cluster, then everybody's lists
    uint64_t list[QLORA_MAX_TOP];        // the block's largest entries in order
    uint32_t group[LP_GROUPS];
    uint32_t bound;
    int count, in_warp[32];
};

// How many logits of the part have a key of at least `least` (the same in every thread).
template <typename T, int THREADS>
__device__ __noinline__ int count_from(const RowParts<T>& row, uint32_t least, TopShared& sh) {
    int n = 0;
    each_from<T, THREADS>(row, least, [&](uint32_t, int) { ++n; });
    __syncthreads();                     // (sh.count has been read by everybody)
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    if ((threadIdx.x & 31) == 0 && n > 0) atomicAdd(&sh.count, n);
    __syncthreads();
    return sh.count;
}

// More candidates than there is room for (many equal logits, or large ones in a cluster): the kk-th largest key itself, found bit by bit
// with a pass over the row each, then everything above it and, in the order of their places, as many equals as are wanted.
template <typename T, int THREADS>
__device__ __noinline__ int crowded(const RowParts<T>& row, int first, int n, int kk, uint32_t bound, TopShared& sh) {
    uint32_t lo = bound, hi = 0xFFFFFFFFu;                          // at least kk keys are >= lo
    while (lo < hi) {                                               // (first whether it is the bound itself: the usual case)
        const uint32_t mid = lo == bound ? bound + 1 : lo + (hi - lo) / 2 + ((hi - lo) & 1);
        if (count_from<T, THREADS>(row, mid, sh) >= kk) lo = mid;
        else hi = mid - 1;
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    if (lo != 0xFFFFFFFFu) each_from<T, THREADS>(row, lo + 1, [&](uint32_t key, int j) { sh.cand[atomicAdd(&sh.count, 1)] = entry_key(key, first + j); });
    __syncthreads();
    int have = sh.count;                                            // fewer than kk
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int j0 = 0; j0 < n && have < kk; j0 += THREADS) {
        const int j = j0 + threadIdx.x;
        const bool is = j < n && order_key(lp_f(row.z[j])) == lo;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, is);
        if (lane == 0) sh.in_warp[warp] = __popc(who);
        __syncthreads();
        int at = have, all = have;
        for (int w = 0; w < THREADS / 32; ++w) {
            at += w < warp ? sh.in_warp[w] : 0;
            all += sh.in_warp[w];
        }
        at += __popc(who & ((1u << lane) - 1u));
        if (is && at < kk) sh.cand[at] = entry_key(lo, first + j);
        have = all;
        __syncthreads();
    }
    return kk;
}

// The kk largest entries of the block's part of the row into sh.list, in order.  `top`: the maximum of this thread's logits.
// The threads fall into groups; at least kk logits are as large as the kk-th largest of the groups' maxima, and few more are (64 groups and kk = 20:
// 24 in the mean).  So only threads with a maximum from there on look at their logits again, which by now are in L2.
template <typename T, int THREADS>
__device__ __forceinline__ void top_of_part(const RowParts<T>& row, int first, int n, int kk, float top, TopShared& sh) {
    const uint32_t key = order_key(top);
    const int groups = kk <= LP_GROUPS / 4 ? LP_GROUPS / 2 : LP_GROUPS, width = THREADS / groups;
    uint32_t g = key;
    for (int o = 1; o < width; o <<= 1) g = max(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
    if (threadIdx.x % width == 0) sh.group[threadIdx.x / width] = g;
    if (threadIdx.x == 0) { sh.bound = 0xFFFFFFFFu; sh.count = 0; }
    __syncthreads();
    if ((int)threadIdx.x < groups) {
        const uint32_t mine = sh.group[threadIdx.x];
        int above = 0;
        for (int q = 0; q < groups; q += 4) {
            const uint4 o = *reinterpret_cast<const uint4*>(&sh.group[q]);
            above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
        const uint32_t least = __reduce_min_sync(0xFFFFFFFFu, above < kk ? mine : 0xFFFFFFFFu);
        if ((threadIdx.x & 31) == 0) atomicMin(&sh.bound, least);
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    if (key >= bound)
        each_from<T, THREADS>(row, bound, [&](uint32_t k, int j) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < LP_CANDIDATES) sh.cand[at] = entry_key(k, first + j);
        });
    __syncthreads();
    int count = sh.count;
    if (count > LP_CANDIDATES) {
        count = crowded<T, THREADS>(row, first, n, kk, bound, sh);
        __syncthreads();
    }
    for (int i = threadIdx.x; i < count; i += THREADS) {             // an entry's place is the number of larger ones
        const uint64_t mine = sh.cand[i];
        int above = 0;
        for (int q = 0; q < count; ++q) above += sh.cand[q] > mine;
        if (above < kk) sh.list[above] = mine;
    }
    __syncthreads();
}

// Shared memory of another block of the cluster.
__device__ __forceinline__ uint32_t remote(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float remote_float(const void* p, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t remote_u64(const void* p, int rank) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
}

// A row to a cluster of `blocks` blocks (1: no cluster), each with a part of it.
template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(int V, long long stride, const T* __restrict__ logits, const int32_t* __restrict__ tokens, float c, int k, int blocks,
                                                           float* __restrict__ logprobs, float* __restrict__ entropy, int32_t* __restrict__ top_ids,
                                                           float* __restrict__ top_logprobs, float* __restrict__ stats) {
    __shared__ RowSums sums[THREADS / 32], mine;
    __shared__ float result[3];
    __shared__ __align__(16) unsigned char top_raw[TOP ? sizeof(TopShared) : 16];
    TopShared& sh = *reinterpret_cast<TopShared*>(top_raw);
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x / blocks, rank = blockIdx.x % blocks, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float kd = c * kLog2e;
    const T* z = logits + row * stride;
    int token = -1;
    float token_logit = 0.f;
    if (threadIdx.x == 0 && rank == 0 && logprobs != nullptr) {
        token = tokens[row];
        if (token >= 0 && token < V) token_logit = lp_f(z[token]);
        else token = -1;
    }
    // the part: whole vectors, but for the row's own ends
    const RowParts<T> whole(z, V);
    auto begin_of = [&](int r) { return r == 0 ? 0 : r == blocks ? V : whole.head + (int)((long long)whole.vectors * r / blocks) * Vec<T>::N; };
    const int first = begin_of(rank), n = begin_of(rank + 1) - first;
    const RowParts<T> part(z + first, n);
    RowSums x = thread_sums<T, THREADS>(part, kd);
    const float top = x.m;
    x = warp_merge(x, kd);
    if (lane == 0) sums[warp] = x;
    if (TOP) top_of_part<T, THREADS>(part, first, n, min(k, n), top, sh);   // (waits for the block)
    else __syncthreads();
    if (warp == 0) {
        x = warp_merge(lane < THREADS / 32 ? sums[lane] : RowSums{-INFINITY, 0.f, 0.f}, kd);
        if (lane == 0) mine = x;
    }
    if (blocks > 1) {
        cluster_sync();
        if (rank == 0 && warp == 0) {
            x = RowSums{-INFINITY, 0.f, 0.f};
            if (lane < blocks) x = RowSums{remote_float(&mine.m, lane), remote_float(&mine.s, lane), remote_float(&mine.a, lane)};
            x = warp_merge(x, kd);
        }
    }
    if (rank == 0 && threadIdx.x == 0) {
        const bool none = x.m == -INFINITY, bad = !(x.m < INFINITY);
        float logs = logf(x.s), H = fmaxf(logs - c * (x.a / x.s), 0.f);
        if (none) { logs = -INFINITY; H = 0.f; }
        if (bad) x.m = logs = H = __int_as_float(0x7FC00000);
        if (stats != nullptr) { stats[3ll * row] = x.m; stats[3ll * row + 1] = logs; stats[3ll * row + 2] = H; }
        if (entropy != nullptr) entropy[row] = H;
        if (logprobs != nullptr) logprobs[row] = token < 0 ? 0.f : none ? -INFINITY : (token_logit - x.m) * c - logs;
        if (TOP) { result[0] = x.m; result[1] = logs; result[2] = none ? 1.f : 0.f; }
    }
    if (TOP && rank == 0) {
        __syncthreads();
        auto put = [&](int at, uint64_t e) {
            if (top_ids != nullptr) top_ids[(long long)row * k + at] = entry_place(e);
            if (top_logprobs != nullptr) top_logprobs[(long long)row * k + at] = result[2] != 0.f ? -INFINITY : (entry_logit(e) - result[0]) * c - result[1];
        };
        if (blocks == 1) {
            if ((int)threadIdx.x < k) put(threadIdx.x, sh.list[threadIdx.x]);
        } else {
            // an entry's place in the whole: its own list's plus, list by list, the number of larger ones
            auto length = [&](int r) { return min(k, begin_of(r + 1) - begin_of(r)); };
            for (int e = threadIdx.x; e < blocks * k; e += THREADS) sh.cand[e] = e % k < length(e / k) ? remote_u64(&sh.list[e % k], e / k) : 0;
            __syncthreads();
            for (int e = threadIdx.x; e < blocks * k; e += THREADS) {
                const uint64_t it = sh.cand[e];
                if (e % k >= length(e / k)) continue;
                int at = e % k;
                for (int r = 0; r < blocks; ++r) {
                    if (r == e / k) continue;
                    int lo = 0, hi = length(r);                      // entries before lo are larger, those from hi on are not
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (sh.cand[r * k + mid] > it) lo = mid + 1; else hi = mid;
                    }
                    at += lo;
                }
                if (at < k) put(at, it);
            }
        }
    }
    if (blocks > 1) cluster_sync();                                  // (nobody leaves while the first block reads)
}

template <typename T>
__global__ void __launch_bounds__(LP_BWD_THREADS) logprobs_bwd_kernel(int V, long long stride, const T* logits, const int32_t* __restrict__ tokens, float c,
                                                                  const float* __restrict__ stats, const float* __restrict__ d_logprobs,
                                                                  const float* __restrict__ d_entropy, long long grad_stride, T* dlogits) {
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x;
    const T* z = logits + row * stride;
    T* dz = dlogits + row * grad_stride;
    const int t = d_logprobs != nullptr ? tokens[row] : -1;
    const float gl = t >= 0 && t < V ? c * d_logprobs[row] : 0.f, gh = d_entropy != nullptr ? c * d_entropy[row] : 0.f;
    const float m = stats[3ll * row], logs = stats[3ll * row + 1], H = stats[3ll * row + 2];
    const bool zero = (gl == 0.f && gh == 0.f) || m == -INFINITY;
    for (int j = threadIdx.x; j < V; j += LP_BWD_THREADS) {
        float g = 0.f;
        if (!zero) {
            const float lp = (lp_f(z[j]) - m) * c - logs, p = expf(lp);
            g = -p * (gl + gh * (fmaxf(lp, -1e30f) + H)) + (j == t ? gl : 0.f);
            if (m != m) g = m;
        }
        dz[j] = lp_to<T>(g);
    }
}

// Blocks that share a row: as many as still fit the SMs all at once, while each has 4 KB of it at least.
static int row_blocks(int T, long long row_bytes, int sms) {
    int blocks = 1;
    while (blocks < LP_CLUSTER && (long long)T * blocks * 2 <= 2 * sms && row_bytes / (blocks * 2) >= 4096) blocks *= 2;
    return blocks;
}

int launch_token_logprobs(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, int k, float* logprobs,
                          float* entropy, int32_t* top_ids, float* top_logprobs, float* stats, cudaStream_t st) {
    const bool top = k > 0;
    const long long row_bytes = (long long)V * (dtype == QLORA_FP32 ? 4 : 2);
    const int blocks = row_blocks(T, row_bytes, sm_count());
    const bool narrow = row_bytes / blocks <= 8192;
    cudaError_t err;
#define QLORA_LP(TYPE, THREADS, TOP)                                                                                                               \
    err = launch_pdl(logprobs_kernel<TYPE, THREADS, TOP>, dim3((unsigned)T * (unsigned)blocks), dim3(THREADS), 0, st, (unsigned)blocks, V, row_stride, \
                     (const TYPE*)logits, tokens, c, k, blocks, logprobs, entropy, top_ids, top_logprobs, stats)
#define QLORA_LP_TYPE(TYPE)                                                                                                                        \
    if (narrow) { if (top) QLORA_LP(TYPE, 128, true); else QLORA_LP(TYPE, 128, false); }                                                            \
    else { if (top) QLORA_LP(TYPE, 512, true); else QLORA_LP(TYPE, 512, false); }
    if (dtype == QLORA_BF16) { QLORA_LP_TYPE(__nv_bfloat16) }
    else if (dtype == QLORA_FP16) { QLORA_LP_TYPE(__half) }
    else { QLORA_LP_TYPE(float) }
#undef QLORA_LP_TYPE
#undef QLORA_LP
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

int launch_token_logprobs_bwd(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, const float* stats,
                              const float* d_logprobs, const float* d_entropy, long long grad_stride, void* dlogits, cudaStream_t st) {
    cudaError_t err;
#define QLORA_LP(TYPE)                                                                                                                              \
    err = launch_pdl(logprobs_bwd_kernel<TYPE>, dim3((unsigned)T), dim3(LP_BWD_THREADS), 0, st, 1, V, row_stride, (const TYPE*)logits, tokens, c, stats,  \
                     d_logprobs, d_entropy, grad_stride, (TYPE*)dlogits)
    if (dtype == QLORA_BF16) QLORA_LP(__nv_bfloat16);
    else if (dtype == QLORA_FP16) QLORA_LP(__half);
    else QLORA_LP(float);
#undef QLORA_LP
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

}  // namespace qlora
