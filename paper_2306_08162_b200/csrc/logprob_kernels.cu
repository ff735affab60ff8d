// Log probabilities of given tokens over [T, V] logits, with each row's entropy and most likely alternatives, and their gradient with
// respect to the logits.  Per row, with c the inverse temperature, m = max z and d_j = c (z_j - m) <= 0:
//     s = sum exp d_j,    log p_j = d_j - log s,    H = log s - (sum exp(d_j) d_j) / s
// in one pass over the row: every thread keeps its own maximum and sums relative to it and corrects them when the maximum moves.
// Bound by HBM in the long run (2 bytes a bf16 logit: 16000 rows of 32000 in 153 us, the time of a copy of as many bytes), by the beginning and end of the
// launch where it is short (888 rows, all that run at a time: 12.6 us; 2048 rows: 26 us, 5.0 TB/s) and, where there are alternatives, by the end of each row, when
// its block has no load on its way: at k = 20 some 9600 of a row's 24700 cycles go to merge, bound, second look and order, with issue 62 % and DRAM 45 % busy
// (k = 32: 36.6 us; 4096 rows of 128000, k = 20: 173 us, 6.1 TB/s).  A logit takes 1 exponential of the special-function unit, whose 16 a
// clock and SM are 57 % busy at 5.1 TB/s, and some 4.5 other instructions: maximum and clamp of two bf16 at once, a fused multiply-add, two sums in pairs.
// The alternatives cost no sorting: see offer_bound.
// Timed and taken out: blocks that stay, with a ring of copies ahead in shared memory (2048 x 32000: 27 - 35 us: fewer warps fit); clusters that share a
// row (one token, k = 20: 8.6 us on 8 blocks, 6.1 then on one); the next round's loads ahead of the sums (26.7 us); 512 or 1024 threads to a row (28, 52 us).
#include "common.cuh"
#include "device_state.h"
#include "f32x2.cuh"
#include "launch.h"

namespace qlora {

constexpr int LP_UNROLL = 4;             // 16-byte vectors that a thread has on their way at a time
constexpr int LP_CANDIDATES = 640;       // entries that are put in order together (a row of less than 64 vectors has fewer logits)
constexpr int LP_HITS = 64;              // stretches that a warp looks at again
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float LP_FLOOR = -0x1p96f, LP_LEAST = -0x1p80f, LP_ODD = 0x1p24f;       // see RowSums

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
    static __device__ __forceinline__ f2 above_floor(const uint4& v, int i) {
        const f2 p = pair(v, i);
        return make_f2(fmaxf(lo_of(p), LP_FLOOR), fmaxf(hi_of(p), LP_FLOOR));
    }
    static __device__ __forceinline__ f2 pair(const uint4& v, int i) { return i == 0 ? make_f2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_f2(__uint_as_float(v.z), __uint_as_float(v.w)); }
    static __device__ __forceinline__ float element(const uint4& v, int i) { return __uint_as_float((i & 2) != 0 ? ((i & 1) != 0 ? v.w : v.z) : ((i & 1) != 0 ? v.y : v.x)); }
    // Bits of the elements that are not below `least` (a NaN is not); element_of(bit) is the element's number.
    static __device__ __forceinline__ uint32_t reaching(const uint4& v, float least) {
        return (__uint_as_float(v.x) < least ? 0u : 1u) | (__uint_as_float(v.y) < least ? 0u : 2u) | (__uint_as_float(v.z) < least ? 0u : 4u) | (__uint_as_float(v.w) < least ? 0u : 8u);
    }
    static __device__ __forceinline__ int element_of(int bit) { return bit; }
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
    static __device__ __forceinline__ float element(const uint4& v, int i) {
        const uint32_t w = word(v, i >> 1);
        return (i & 1) != 0 ? bf16_hi(w) : bf16_lo(w);
    }
    typedef __nv_bfloat162 Max;
    static __device__ __forceinline__ f2 above_floor(const uint4& v, int i) {            // (both at once, as they lie in memory)
        const Max m = __hmax2(of(word(v, i)), __float2bfloat162_rn(LP_FLOOR));
        return unpack_bf16(*reinterpret_cast<const uint32_t*>(&m));
    }
    static __device__ __forceinline__ Max lowest() { return __float2bfloat162_rn(-INFINITY); }
    static __device__ __forceinline__ Max of(uint32_t w) { return *reinterpret_cast<const Max*>(&w); }
    // (two elements at once; the upper ones of the pairs are 16 bits up)
    static __device__ __forceinline__ uint32_t reaching(const uint4& v, float least) {
        const Max b = __float2bfloat162_rn(least);
        return (~__hlt2_mask(of(v.x), b) & 0x00020001u) | (~__hlt2_mask(of(v.y), b) & 0x00080004u) | (~__hlt2_mask(of(v.z), b) & 0x00200010u) | (~__hlt2_mask(of(v.w), b) & 0x00800040u);
    }
    static __device__ __forceinline__ int element_of(int bit) { return bit & 15; }
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
    static __device__ __forceinline__ float element(const uint4& v, int i) { return __half2float(__ushort_as_half((unsigned short)(word(v, i >> 1) >> (16 * (i & 1))))); }
    static __device__ __forceinline__ f2 above_floor(const uint4& v, int i) {
        const f2 p = pair(v, i);
        return make_f2(fmaxf(lo_of(p), LP_FLOOR), fmaxf(hi_of(p), LP_FLOOR));
    }
    typedef __half2 Max;
    static __device__ __forceinline__ Max lowest() { return __float2half2_rn(-INFINITY); }
    static __device__ __forceinline__ Max of(uint32_t w) { return *reinterpret_cast<const Max*>(&w); }
    // (two elements at once; the upper ones of the pairs are 16 bits up)
    static __device__ __forceinline__ uint32_t reaching(const uint4& v, float least) {
        const Max b = __float2half2_rn(least);
        return (~__hlt2_mask(of(v.x), b) & 0x00020001u) | (~__hlt2_mask(of(v.y), b) & 0x00080004u) | (~__hlt2_mask(of(v.z), b) & 0x00200010u) | (~__hlt2_mask(of(v.w), b) & 0x00800040u);
    }
    static __device__ __forceinline__ int element_of(int bit) { return bit & 15; }
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

// 16 bytes that are read once.  asm volatile: several loads stay ahead of their uses.
template <bool KEEP = false>
__device__ __forceinline__ uint4 load_stream(const uint4* p) {          // KEEP: in L1, for a second look
    uint4 v;
    if (KEEP) asm volatile("ld.global.L1::evict_last.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    else asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
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
__device__ __forceinline__ float key_logit(uint32_t key) {
    return key == 0xFFFFFFFFu ? __int_as_float(0x7FC00000) : __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ float entry_logit(uint64_t e) { return key_logit((uint32_t)(e >> 32)); }

// A maximum m and sums relative to it in base 2: with kd = c log2(e) and r = m kd as it is rounded,
//     s = sum 2^x_j,   a = sum 2^x_j x_j,   x_j = z_j kd - r   (one fused multiply-add: an error of half a place of x_j, not of z_j kd)
// For that 2^-30 <= c <= 2^30, logits below LP_FLOOR count as that (-inf among them: 2^x is 0 and 2^x x is 0, not NaN), and r is at least
// LP_LEAST kd.  The maximum's own x is the rounding error of r, half a place of m kd: below LP_ODD = 2^24 at most a half, but 128 and more from 2^31 on, where
// 2^x leaves fp32's range.  Rows with |m| kd from LP_ODD on are summed again from the differences (odd_row).  A thread whose own maximum is that large
// in a row that is not (masked logits) may hold infinite sums: its maximum lies far enough below the row's for rebase to drop them.
struct RowSums {
    float m, s, a;
};
__device__ __forceinline__ float reference(float m, float kd) { return __fmul_rn(fmaxf(m, LP_LEAST), kd); }   // (rounded by itself: the differences of two rely on it)
// Moves the sums to a maximum m >= x.m.
__device__ __forceinline__ void rebase(RowSums& x, float m, float kd) {
    const float shift = reference(x.m, kd) - reference(m, kd), e = fast_exp2(shift);
    x.a = e > 0.f ? e * fmaf(x.s, shift, x.a) : 0.f;
    x.s = e > 0.f ? x.s * e : 0.f;
    x.m = m;
}
__device__ __forceinline__ void add_one(RowSums& x, float z, float kd) {
    const float m = max_nan(x.m, z);
    if (m != x.m) rebase(x, m, kd);
    const float y = fmaf(fmaxf(z, LP_FLOOR), kd, -reference(m, kd)), e = fast_exp2(y);
    x.s += e;
    x.a = fmaf(e, y, x.a);
}
// The largest of a warp's values, NaN if one of them is (one reduction of whole numbers instead of five exchanges).
__device__ __forceinline__ float warp_max_nan(float m) { return key_logit(__reduce_max_sync(0xFFFFFFFFu, order_key(m))); }
// Sums over LANES lanes of a warp that are next to each other, relative to their common maximum m, the same in all of them.
template <int LANES>
__device__ __forceinline__ RowSums merged(RowSums x, float m, float kd) {
    rebase(x, m, kd);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        x.s += __shfl_xor_sync(0xFFFFFFFFu, x.s, o);
        x.a += __shfl_xor_sync(0xFFFFFFFFu, x.a, o);
    }
    return x;
}

// log s and the entropy of a row whose maximum m is finite but too far from zero for the sums above (a row masked altogether by a large negative number,
// a temperature near zero): from the differences to m themselves, by the whole block.
// (Logit by logit: 2048 such rows of 32000 take 69 us.)
template <typename T, int THREADS>
__device__ __noinline__ void odd_row(const T* z, int V, float m, float c, float* sums, float& logs, float& H) {
    float s = 0.f, a = 0.f;
    for (int j = threadIdx.x; j < V; j += THREADS) {
        const float d = fmaxf((lp_f(z[j]) - m) * c, -1e30f), e = expf(d);
        s += e;
        a = fmaf(e, d, a);
    }
    s = warp_sum(s);
    a = warp_sum(a);
    if ((threadIdx.x & 31) == 0) { sums[2 * (threadIdx.x >> 5)] = s; sums[2 * (threadIdx.x >> 5) + 1] = a; }
    __syncthreads();
    s = a = 0.f;
    for (int w = 0; w < THREADS / 32; ++w) { s += sums[2 * w]; a += sums[2 * w + 1]; }
    logs = logf(s);
    H = fmaxf(logs - a / s, 0.f);
}

// This thread's part of a row, LP_UNROLL vectors (a round) at a time.  TOP: the maximum of each stretch of 2^span_log2 rounds goes to segment[stretch].
// (SINGLE: every round is one.)
template <typename T, int THREADS, bool TOP, bool SINGLE>
struct ThreadRow {
    RowSums x;
    float stretch;
    float* segment;
    int left, span;
    __device__ __forceinline__ ThreadRow(float* segments, int span_log2) : x{-INFINITY, 0.f, 0.f}, stretch(-INFINITY), segment(segments), left(1 << span_log2), span(1 << span_log2) {}
    // Vector u of the round is there where c0 + u * THREADS < vectors.
    template <bool WHOLE>
    __device__ __forceinline__ void round(const uint4 (&v)[LP_UNROLL], int c0, int vectors, float kd) {
        typename Vec<T>::Max top = Vec<T>::lowest();
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (WHOLE || c0 + u * THREADS < vectors) top = Vec<T>::fold(top, v[u]);
        const float here = Vec<T>::value(top), m = max_nan(x.m, here);
        if (TOP && SINGLE) *segment++ = here;
        if (TOP && !SINGLE) {
            stretch = max_nan(stretch, here);
            if (--left == 0) {
                *segment++ = stretch;
                stretch = -INFINITY;
                left = span;
            }
        }
        if (m != x.m) rebase(x, m, kd);
        const float r = reference(m, kd);
        const f2 minus_r = make_f2(-r, -r), kd2 = make_f2(kd, kd);
        f2 s2 = make_f2(x.s, 0.f), a2 = make_f2(x.a, 0.f);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (WHOLE || c0 + u * THREADS < vectors) {
#pragma unroll
                for (int i = 0; i < Vec<T>::N / 2; ++i) {
                    const f2 y = fma2(Vec<T>::above_floor(v[u], i), kd2, minus_r), e = exp2_2(y);
                    s2 = add2(s2, e);
                    a2 = fma2(e, y, a2);
                }
            }
        x.s = lo_of(s2) + hi_of(s2);
        x.a = lo_of(a2) + hi_of(a2);
    }
    __device__ __forceinline__ void finish() {
        if (TOP && !SINGLE && left != span) *segment = stretch;
    }
};

// Calls f(key, place) for this thread's logits whose key is at least `least`.
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

struct alignas(16) TopShared {              // (the candidates are read two at a time)
    uint64_t cand[LP_CANDIDATES];        // entries that may be among the largest
    uint32_t bound[32], next[32];        // by warp (of those that stay out: the largest key, and 0)
    int count, more, in_warp[32];
};
template <int THREADS, int SEGMENTS> struct alignas(16) TopWarps {
    static constexpr int STRIDE = SEGMENTS == 4 ? 4 : SEGMENTS + 4;          // (16 bytes at a time, and fewer in the same bank)
    float segment[THREADS * STRIDE];         // maxima of the threads' stretches
    int hit[THREADS / 32][LP_HITS];         // stretches with a candidate, by their first vector
};

// How many logits of the row have a key of at least `least` (the same in every thread).
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

// More candidates than there is room for (many equal logits, as where fewer than kk are unmasked, or large ones close together): the kk-th largest key
// itself, halving what is left by a pass over the row each time, then everything above it and, in the order of their places, as many equals as are wanted.
template <typename T, int THREADS>
__device__ __noinline__ int crowded(const RowParts<T>& row, int n, int kk, uint32_t bound, TopShared& sh) {
    uint32_t lo = bound, hi = 0xFFFFFFFFu;                          // at least kk keys are >= lo
    while (lo < hi) {                                               // (first whether it is the bound itself: the usual case)
        const uint32_t mid = lo == bound ? bound + 1 : lo + (hi - lo) / 2 + ((hi - lo) & 1);
        if (count_from<T, THREADS>(row, mid, sh) >= kk) lo = mid;
        else hi = mid - 1;
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    if (lo != 0xFFFFFFFFu) each_from<T, THREADS>(row, lo + 1, [&](uint32_t key, int j) { sh.cand[atomicAdd(&sh.count, 1)] = entry_key(key, j); });
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
        if (is && at < kk) sh.cand[at] = entry_key(lo, j);
        have = all;
        __syncthreads();
    }
    return kk;
}

// The alternatives.  kk = q warps + r: at least kk logits of the row are as large as both the smallest of the warps' q-th largest lane maxima and the r-th largest
// of their next ones, and not many more are (256 threads and kk = 20: some 40 in the mean), so these are found again and put in order, and nothing else
// is done for the others.
// Here, before the block waits: what this warp gives to that bound.  `top`: the maximum of this thread's logits.  Warps that lack logits stay out of it.
template <int THREADS>
__device__ __forceinline__ void offer_bound(int vectors, int kk, float top, TopShared& sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = min(THREADS / 32, vectors / 32);
    uint32_t key = order_key(top), least = 0xFFFFFFFFu, next = 0;
    int more = 0;
    if (warps * 32 < kk) least = 0;                                  // (a short row: everything is a candidate)
    else if (warp < warps) {
        for (int q = kk; q > 0; q -= warps) {
            next = __reduce_max_sync(0xFFFFFFFFu, key);
            if (q < warps) {                                         // (r more from one warp or another)
                more = q;
                break;
            }
            least = next;
            if (lane == __ffs(__ballot_sync(0xFFFFFFFFu, key == least)) - 1) key = 0;
        }
    }
    if (lane == 0) {
        sh.bound[warp] = least;
        sh.next[warp] = next;
    }
    if (threadIdx.x == 0) {
        sh.count = 0;
        sh.more = more;
    }
}
template <int THREADS>
__device__ __forceinline__ uint32_t common_bound(const TopShared& sh) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, r = sh.more;
    uint32_t bound = sh.bound[lane & (WARPS - 1)];
    if (r > 0 && lane < WARPS) {                                     // (the r largest of the next ones: fewer than r are above)
        const uint32_t mine = sh.next[lane];
        int above = 0;
#pragma unroll
        for (int w = 0; w < WARPS; w += 2) {
            const uint2 two = *reinterpret_cast<const uint2*>(&sh.next[w]);
            above += (two.x > mine) + (two.y > mine);
        }
        if (above < r) bound = min(bound, mine);
    }
    return __reduce_min_sync(0xFFFFFFFFu, bound);
}

// After it: the entries from the bound on.  Each warp looks again at the stretches of its own lanes that reach it; their logits are in L1 or L2 by now.
// `segment`: the maxima of this thread's stretches; `hit`: LP_HITS places of this warp's own; head, rest: the logits at this thread's places there.
// meanwhile(): work of the warp that does not depend on the loads.
template <typename T, int THREADS, int SEGMENTS, typename F>
__device__ __forceinline__ void gather(const RowParts<T>& row, uint32_t bound, int span_log2, const float* segment, int* hit, float head, float rest, TopShared& sh, F meanwhile) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t below = (1u << lane) - 1u;
    // the stretches of this lane that reach the bound, as bits
    const float least = key_logit(bound);
    constexpr int ROUND_LOG2 = THREADS == 64 ? 8 : THREADS == 128 ? 9 : THREADS == 256 ? 10 : 11;
    static_assert(1 << ROUND_LOG2 == LP_UNROLL * THREADS, "vectors of a round");
    const int stretch_log2 = ROUND_LOG2 + span_log2, stretches = (max(row.vectors - (int)threadIdx.x, 0) + (1 << stretch_log2) - 1) >> stretch_log2;
    uint32_t reach = 0;
#pragma unroll
    for (int g = 0; g < SEGMENTS; g += 4) {
        if (g > 0 && g >= stretches) break;
        const float4 four = *reinterpret_cast<const float4*>(segment + g);
        if (!(four.x < least)) reach |= 1u << g;
        if (!(four.y < least)) reach |= 2u << g;
        if (!(four.z < least)) reach |= 4u << g;
        if (!(four.w < least)) reach |= 8u << g;
    }
    reach &= (1u << stretches) - 1u;
    int hits = 0;
    for (uint32_t who; (who = __ballot_sync(0xFFFFFFFFu, reach != 0)) != 0; hits += __popc(who)) {
        if (reach == 0) continue;
        const int at = hits + __popc(who & below), g = __ffs(reach) - 1;
        if (at < LP_HITS) hit[at] = threadIdx.x + (g << stretch_log2);
        reach &= reach - 1;
    }
    if (hits > LP_HITS || bound == 0xFFFFFFFFu) {                    // (each has a candidate; kk NaN)
        if (lane == 0) atomicAdd(&sh.count, LP_CANDIDATES + 1);
        hits = 0;
    }
    __syncwarp();
    auto put = [&](int at, uint32_t key, int j) {
        if (at < LP_CANDIDATES) sh.cand[at] = entry_key(key, j);
    };
    static_assert(LP_UNROLL == 4, "the vectors of a stretch are a power of two");
    const int work = hits << (span_log2 + 2);
    if (work == 0) meanwhile();
    for (int w0 = 0; w0 < work; w0 += 32) {
        const int w = w0 + lane, at = w < work ? hit[w >> (span_log2 + 2)] + (w & ((LP_UNROLL << span_log2) - 1)) * THREADS : row.vectors;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (at < row.vectors) v = load_stream<true>(row.body() + at);
        if (w0 == 0) meanwhile();
        uint32_t found = at < row.vectors ? Vec<T>::reaching(v, least) : 0;
        for (; found != 0; found &= found - 1) {
            const int i = Vec<T>::element_of(__ffs(found) - 1);
            put(atomicAdd(&sh.count, 1), order_key(Vec<T>::element(v, i)), row.head + at * Vec<T>::N + i);
        }
    }
    if ((int)threadIdx.x < row.head && order_key(head) >= bound) put(atomicAdd(&sh.count, 1), order_key(head), threadIdx.x);
    if ((int)threadIdx.x < row.rest && order_key(rest) >= bound) put(atomicAdd(&sh.count, 1), order_key(rest), row.tail + threadIdx.x);
}

// With the candidates there (behind a barrier): calls put(place, entry) for the kk largest.
template <typename T, int THREADS, int LANES, typename F>
__device__ __forceinline__ void select(const RowParts<T>& row, int n, int kk, uint32_t bound, TopShared& sh, F put) {
    int count = sh.count;
    if (count > LP_CANDIDATES) {
        count = crowded<T, THREADS>(row, n, kk, bound, sh);
        __syncthreads();
    }
    // An entry's place is the number of larger ones, which LANES lanes count a part of each.
    const int part = threadIdx.x % LANES, warp = threadIdx.x >> 5;
    for (int i0 = warp * (32 / LANES); i0 < count; i0 += THREADS / LANES) {
        const int i = i0 + (threadIdx.x & 31) / LANES;
        const uint64_t mine = sh.cand[min(i, count - 1)];
        int above = 0;
        for (int q = 2 * part; q + 1 < count; q += 2 * LANES) {
            const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sh.cand[q]);
            above += (two.x > mine) + (two.y > mine);
        }
        if ((count & 1) && part == 0) above += sh.cand[count - 1] > mine;
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) above += __shfl_xor_sync(0xFFFFFFFFu, above, o);
        if (part == 0 && i < count && above < kk) put(above, mine);
    }
}

struct LogprobArgs {
    int T, V, k;
    long long stride;
    const void* logits;
    const int32_t* tokens;
    float c;
    float *logprobs, *entropy, *stats, *top_logprobs;
    int32_t* top_ids;
};

// What one thread that has a row's sums tells about it; the result is what the alternatives need.
struct RowResult {
    float m, logs;
    int none;
};
__device__ __forceinline__ RowResult tell_row(const LogprobArgs& p, int row, RowSums x, float kd, bool odd, float logs, float H, int token, float token_logit) {
    const bool none = x.m == -INFINITY;
    if (!odd) {
        const float ln_s = logf(x.s);
        logs = fmaxf(fmaf(fmaf(-x.m, kd, reference(x.m, kd)), kLn2, ln_s), 0.f);   // (a sum relative to the maximum is at least 1)
        H = fmaxf(ln_s - kLn2 * __fdividef(x.a, x.s), 0.f);
        if (none) { logs = -INFINITY; H = 0.f; }
        if (!(x.m < INFINITY)) x.m = logs = H = __int_as_float(0x7FC00000);
    }
    if (p.stats != nullptr) { p.stats[3ll * row] = x.m; p.stats[3ll * row + 1] = logs; p.stats[3ll * row + 2] = H; }
    if (p.entropy != nullptr) p.entropy[row] = H;
    if (p.logprobs != nullptr) p.logprobs[row] = token < 0 ? 0.f : none ? -INFINITY : (token_logit - x.m) * p.c - logs;
    return RowResult{x.m, logs, none};
}
__device__ __forceinline__ void tell_top(const LogprobArgs& p, int row, int at, uint64_t e, const RowResult& r) {
    if (p.top_ids != nullptr) p.top_ids[(long long)row * p.k + at] = entry_place(e);
    if (p.top_logprobs != nullptr) p.top_logprobs[(long long)row * p.k + at] = r.none ? -INFINITY : (entry_logit(e) - r.m) * p.c - r.logs;
}
__device__ __forceinline__ bool is_odd(float m, float kd) { return fabsf(m) < INFINITY && !(fabsf(m) * kd < LP_ODD); }
template <int THREADS, int SEGMENTS>
__device__ __forceinline__ int span_of(int vectors) {                    // log2 of the rounds that make a stretch
    const int round = LP_UNROLL * THREADS, rounds = (vectors + round - 1) / round;
    return rounds <= SEGMENTS ? 0 : 32 - __clz((rounds - 1) / SEGMENTS);
}

// How a row is shared out.  What a row costs beside its logits goes with the warps that share it, so they are as few as its length allows:
//                                      64 threads    128 threads    256 threads
//   8192 rows of 4000 bf16, k = 5         26 us         35 us           -
//   4000 rows of 10000, k = 20             -            28 us          38 us
//   2048 rows of 32000, k = 32             -            53 us          37 us       (fewer warps than hide the loads' latency)
// and 512 where all rows run at a time even so, three to an SM (300 rows of 128000, k = 20: 24.6 us, with 256 threads 29.6; 300 of 32000, k = 0: 6.4, with 256
// 7.6; with alternatives rows of up to 64 KB gain at some numbers and lose at others: 200 of 32000, k = 20: 11.2, with 256 12.7; 296: 12.4 and 9.9), or an SM to
// every row, with the next round's loads ahead (one row of 32000, k = 20: 5.9 us).
// SINGLE: a row has so few rounds that each is a stretch.  KEEP: the row stays in L1 for the second look at it (2048 rows of 32000, k = 32: 36.9 us,
// without 39.3; rows of 200 KB: 48 us, without 45).
struct TinyRow { static constexpr int THREADS = 64, SEGMENTS = 4, PER_SM = 20; static constexpr bool SINGLE = true, AHEAD = false, KEEP = true; };
struct ShortRow { static constexpr int THREADS = 128, SEGMENTS = 4, PER_SM = 10; static constexpr bool SINGLE = true, AHEAD = false, KEEP = true; };
struct MiddleRow { static constexpr int THREADS = 256, SEGMENTS = 4, PER_SM = 6; static constexpr bool SINGLE = true, AHEAD = false, KEEP = true; };
struct LongRow { static constexpr int THREADS = 256, SEGMENTS = 16, PER_SM = 6; static constexpr bool SINGLE = false, AHEAD = false, KEEP = false; };
struct FewRow { static constexpr int THREADS = 512, SEGMENTS = 8, PER_SM = 3; static constexpr bool SINGLE = false, AHEAD = false, KEEP = false; };
struct LoneRow { static constexpr int THREADS = 512, SEGMENTS = 8, PER_SM = 1; static constexpr bool SINGLE = false, AHEAD = true, KEEP = true; };

template <typename T, typename Plan, bool TOP>
__global__ void __launch_bounds__(Plan::THREADS, Plan::PER_SM) logprobs_kernel(const __grid_constant__ LogprobArgs p) {
    constexpr int THREADS = Plan::THREADS, SEGMENTS = Plan::SEGMENTS;
    constexpr bool KEEP = TOP && Plan::KEEP;
    __shared__ RowSums sums[THREADS / 32];
    __shared__ RowResult result;
    __shared__ float odd_sums[2 * (THREADS / 32)];
    __shared__ __align__(16) unsigned char top_raw[TOP ? sizeof(TopShared) : 16], warps_raw[TOP ? sizeof(TopWarps<THREADS, SEGMENTS>) : 16];
    TopShared& sh = *reinterpret_cast<TopShared*>(top_raw);
    TopWarps<THREADS, SEGMENTS>& own = *reinterpret_cast<TopWarps<THREADS, SEGMENTS>*>(warps_raw);
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, V = p.V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float kd = p.c * kLog2e;
    const T* z = static_cast<const T*>(p.logits) + row * p.stride;
    const RowParts<T> part(z, V);
    const int token = threadIdx.x == 0 && p.logprobs != nullptr ? p.tokens[row] : -1;
    const float head = (int)threadIdx.x < part.head ? lp_f(part.z[threadIdx.x]) : -INFINITY;
    const float rest = (int)threadIdx.x < part.rest ? lp_f(part.z[part.tail + threadIdx.x]) : -INFINITY;
    const int span_log2 = Plan::SINGLE ? 0 : span_of<THREADS, SEGMENTS>(part.vectors);
    ThreadRow<T, THREADS, TOP, Plan::SINGLE> mine(own.segment + own.STRIDE * threadIdx.x, span_log2);
    int c0 = threadIdx.x;
    if (Plan::AHEAD) {                                                // the next round's vectors are on their way while one is summed
        uint4 v[LP_UNROLL], w[LP_UNROLL];
        auto load = [&](uint4 (&to)[LP_UNROLL], int c) {
#pragma unroll
            for (int u = 0; u < LP_UNROLL; ++u)
                if (c + u * THREADS < part.vectors) to[u] = load_stream<KEEP>(part.body() + c + u * THREADS);
        };
        load(v, c0);
        for (; c0 < part.vectors; c0 += LP_UNROLL * THREADS) {
            load(w, c0 + LP_UNROLL * THREADS);
            mine.template round<false>(v, c0, part.vectors, kd);
#pragma unroll
            for (int u = 0; u < LP_UNROLL; ++u) v[u] = w[u];
        }
    }
    for (; c0 + (LP_UNROLL - 1) * THREADS < part.vectors; c0 += LP_UNROLL * THREADS) {
        uint4 v[LP_UNROLL];
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) v[u] = load_stream<KEEP>(part.body() + c0 + u * THREADS);
        mine.template round<true>(v, c0, part.vectors, kd);
    }
    if (c0 < part.vectors) {
        uint4 v[LP_UNROLL];
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * THREADS < part.vectors) v[u] = load_stream<KEEP>(part.body() + c0 + u * THREADS);
        mine.template round<false>(v, c0, part.vectors, kd);
    }
    mine.finish();
    const float token_logit = token >= 0 && token < V ? lp_f(z[token]) : 0.f;
    if ((int)threadIdx.x < part.head) add_one(mine.x, head, kd);
    if ((int)threadIdx.x < part.rest) add_one(mine.x, rest, kd);
    if (TOP) offer_bound<THREADS>(part.vectors, p.k, mine.x.m, sh);
    RowSums x = merged<32>(mine.x, warp_max_nan(mine.x.m), kd);
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    // One warp tells about the row; where its maximum is odd, all of them sum it again first.
    auto tell = [&](bool odd, float logs, float H) {
        if (warp != 0) return;
        if (!odd) {
            x = sums[lane & (THREADS / 32 - 1)];
            x = merged<THREADS / 32>(x, warp_max_nan(x.m), kd);
        }
        if (lane == 0) result = tell_row(p, row, x, kd, odd, logs, H, token >= 0 && token < V ? token : -1, token_logit);
    };
    auto tell_odd = [&]() {
        float logs, H;
        odd_row<T, THREADS>(z, V, result.m, p.c, odd_sums, logs, H);
        tell(true, logs, H);
    };
    if (TOP) {
        const uint32_t bound = common_bound<THREADS>(sh);
        gather<T, THREADS, SEGMENTS>(part, bound, span_log2, own.segment + own.STRIDE * threadIdx.x, own.hit[warp], head, rest, sh, [&]() { tell(false, 0.f, 0.f); });
        __syncthreads();
        if (is_odd(result.m, kd)) {
            tell_odd();
            __syncthreads();
        }
        select<T, THREADS, Plan::AHEAD ? 4 : 1>(part, V, p.k, bound, sh, [&](int at, uint64_t e) { tell_top(p, row, at, e, result); });
    } else {
        tell(false, 0.f, 0.f);
        if (is_odd(warp_max_nan(sums[lane & (THREADS / 32 - 1)].m), kd)) {
            __syncthreads();
            tell_odd();
        }
    }
}

// Gradient.  With the row's statistics a logit's gradient needs nothing but the logit: p = 2^x, x = (z - m) kd - log2 s, and
//     dz = -p ((gl + gh H) + gh ln 2 x)  (+ gl at the token),   gl = c d_logprobs, gh = c d_entropy.
// Bound by HBM (each logit read once, each gradient written once): 2048 x 32000 bf16 in 42.7 us, 6.1 TB/s.  A block has two vectors of a row
// per thread and 8 blocks share an SM: with four vectors long rows take the same (42.6 us), 8192 rows of 4000 23.4 us instead of 21.4.
struct BwdArgs {
    int T, V;
    long long stride, grad_stride;
    const void* logits;
    const int32_t* tokens;
    float c;
    const float *stats, *d_logprobs, *d_entropy;
    void* dlogits;
};

struct RowGradient {
    float m, log2_s, base, per_x, gl, kd;                             // dz = -p (base + per_x x)
    int token;
    bool zero, broken;
    __device__ __forceinline__ RowGradient(const BwdArgs& p, int row) {
        token = p.d_logprobs != nullptr ? p.tokens[row] : -1;
        gl = p.d_logprobs != nullptr ? p.d_logprobs[row] : 0.f;
        const float gh = p.d_entropy != nullptr ? p.c * p.d_entropy[row] : 0.f, H = p.stats[3ll * row + 2];
        m = p.stats[3ll * row];
        log2_s = p.stats[3ll * row + 1] * kLog2e;
        if (token < 0 || token >= p.V) { token = -1; gl = 0.f; }
        gl *= p.c;
        kd = p.c * kLog2e;
        base = fmaf(gh, H, gl);
        per_x = gh * kLn2;
        zero = (gl == 0.f && gh == 0.f) || m == -INFINITY;
        broken = m != m;
    }
    // (below 2^-256 a probability is 0; the logarithm of a masked one is kept finite, so that their product is 0 too)
    template <bool ENTROPY>
    __device__ __forceinline__ f2 of_pair(f2 z) const {
        const f2 x = fma2(add2(z, make_f2(-m, -m)), make_f2(kd, kd), make_f2(-log2_s, -log2_s));
        if (!ENTROPY) return mul2(exp2_2(x), make_f2(-base, -base));
        const f2 y = make_f2(fmaxf(lo_of(x), -256.f), fmaxf(hi_of(x), -256.f));
        return mul2(exp2_2(y), fma2(y, make_f2(-per_x, -per_x), make_f2(-base, -base)));
    }
    __device__ __forceinline__ float of_one(float z, int j) const {
        if (broken) return m;
        const f2 g = of_pair<true>(make_f2(z, z));
        return lo_of(g) + (j == token ? gl : 0.f);
    }
};

template <typename T> __device__ __forceinline__ uint32_t pack_pair(f2 g);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(f2 g) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo_of(g), hi_of(g));
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(f2 g) {
    const __half2 v = __floats2half2_rn(lo_of(g), hi_of(g));
    return *reinterpret_cast<const uint32_t*>(&v);
}

template <typename T, bool ENTROPY>
__device__ __forceinline__ uint4 gradient_of(const RowGradient& r, const uint4& v, int token_at) {
    f2 g[Vec<T>::N / 2];
#pragma unroll
    for (int i = 0; i < Vec<T>::N / 2; ++i) g[i] = r.template of_pair<ENTROPY>(Vec<T>::pair(v, i));
    if ((unsigned)token_at < (unsigned)Vec<T>::N) {
#pragma unroll
        for (int i = 0; i < Vec<T>::N / 2; ++i) g[i] = add2(g[i], make_f2(token_at == 2 * i ? r.gl : 0.f, token_at == 2 * i + 1 ? r.gl : 0.f));
    }
    if constexpr (Vec<T>::N == 4) return make_uint4(__float_as_uint(lo_of(g[0])), __float_as_uint(hi_of(g[0])), __float_as_uint(lo_of(g[1])), __float_as_uint(hi_of(g[1])));
    else return make_uint4(pack_pair<T>(g[0]), pack_pair<T>(g[1]), pack_pair<T>(g[2]), pack_pair<T>(g[3]));
}

constexpr int LP_BWD_UNROLL = 2, LP_BWD_THREADS = 256;

// Rows of logits and gradient that begin at the same place within 16 bytes.  grid: (rows, stretches of a row).
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(LP_BWD_THREADS, 8) logprobs_bwd_kernel(const __grid_constant__ BwdArgs p) {
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, c0 = blockIdx.y * (LP_BWD_UNROLL * LP_BWD_THREADS) + threadIdx.x;
    const RowGradient r(p, row);
    const RowParts<T> part(static_cast<const T*>(p.logits) + row * p.stride, p.V);
    T* dz = static_cast<T*>(p.dlogits) + row * p.grad_stride;
    uint4* body = reinterpret_cast<uint4*>(dz + part.head);
    if (r.zero || r.broken) {
        const float g = r.zero ? 0.f : r.m;
        uint4 all;
        if constexpr (sizeof(T) == 4) all.x = __float_as_uint(g);
        else all.x = pack_pair<T>(make_f2(g, g));
        all.y = all.z = all.w = all.x;
#pragma unroll
        for (int u = 0; u < LP_BWD_UNROLL; ++u)
            if (c0 + u * LP_BWD_THREADS < part.vectors) __stcs(body + c0 + u * LP_BWD_THREADS, all);
        if (blockIdx.y == 0) {
            if ((int)threadIdx.x < part.head) dz[threadIdx.x] = lp_to<T>(g);
            if ((int)threadIdx.x < part.rest) dz[part.tail + threadIdx.x] = lp_to<T>(g);
        }
        return;
    }
    uint4 v[LP_BWD_UNROLL];
#pragma unroll
    for (int u = 0; u < LP_BWD_UNROLL; ++u)
        if (c0 + u * LP_BWD_THREADS < part.vectors) v[u] = load_stream(part.body() + c0 + u * LP_BWD_THREADS);
    const int token_vector = r.token - part.head;                      // (negative without one)
#pragma unroll
    for (int u = 0; u < LP_BWD_UNROLL; ++u)
        if (c0 + u * LP_BWD_THREADS < part.vectors) __stcs(body + c0 + u * LP_BWD_THREADS, gradient_of<T, ENTROPY>(r, v[u], token_vector - (c0 + u * LP_BWD_THREADS) * Vec<T>::N));
    if (blockIdx.y == 0) {
        if ((int)threadIdx.x < part.head) dz[threadIdx.x] = lp_to<T>(r.of_one(lp_f(part.z[threadIdx.x]), threadIdx.x));
        const int j = part.tail + threadIdx.x;
        if ((int)threadIdx.x < part.rest) dz[j] = lp_to<T>(r.of_one(lp_f(part.z[j]), j));
    }
}

// Rows that begin at different places: one logit at a time, 2 bytes a load (2048 x 32000 bf16: 138 us, where rows that begin alike take 44).
template <typename T>
__global__ void __launch_bounds__(LP_BWD_THREADS) logprobs_bwd_scalar_kernel(const __grid_constant__ BwdArgs p) {
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x;
    const RowGradient r(p, row);
    const T* z = static_cast<const T*>(p.logits) + row * p.stride;
    T* dz = static_cast<T*>(p.dlogits) + row * p.grad_stride;
    const int begin = blockIdx.y * (LP_BWD_UNROLL * LP_BWD_THREADS * Vec<T>::N), end = min(p.V, begin + LP_BWD_UNROLL * LP_BWD_THREADS * Vec<T>::N);
    for (int j = begin + threadIdx.x; j < end; j += LP_BWD_THREADS) dz[j] = lp_to<T>(r.zero ? 0.f : r.of_one(lp_f(z[j]), j));
}

template <typename T, typename Plan>
static cudaError_t launch_logprobs_as(const LogprobArgs& p, cudaStream_t st) {
    const dim3 grid((unsigned)p.T), block(Plan::THREADS);
    return p.k > 0 ? launch_pdl(logprobs_kernel<T, Plan, true>, grid, block, 0, st, 1, p) : launch_pdl(logprobs_kernel<T, Plan, false>, grid, block, 0, st, 1, p);
}
template <typename T>
static cudaError_t launch_logprobs(const LogprobArgs& p, cudaStream_t st) {
    const long long row_bytes = (long long)p.V * (int)sizeof(T);
    const int sms = sm_count();
    // (64 threads: their 64 maxima bound up to 32 alternatives well, and it takes more rows than 20 blocks an SM to gain)
    if (row_bytes <= 8 << 10 && p.k <= 32 && p.T > 20 * sms) return launch_logprobs_as<T, TinyRow>(p, st);
    if (row_bytes <= 8 << 10 || (row_bytes <= 32 << 10 && p.T > sms)) return launch_logprobs_as<T, ShortRow>(p, st);
    if (p.T <= sms) return launch_logprobs_as<T, LoneRow>(p, st);
    if (p.T <= FewRow::PER_SM * sms && (p.k == 0 || row_bytes > 64 << 10)) return launch_logprobs_as<T, FewRow>(p, st);
    if (row_bytes <= 64 << 10) return launch_logprobs_as<T, MiddleRow>(p, st);
    return launch_logprobs_as<T, LongRow>(p, st);
}

int launch_token_logprobs(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, int k, float* logprobs,
                          float* entropy, int32_t* top_ids, float* top_logprobs, float* stats, cudaStream_t st) {
    const LogprobArgs p{T, V, k, row_stride, logits, tokens, c, logprobs, entropy, stats, top_logprobs, top_ids};
    const cudaError_t err = dtype == QLORA_BF16 ? launch_logprobs<__nv_bfloat16>(p, st) : dtype == QLORA_FP16 ? launch_logprobs<__half>(p, st) : launch_logprobs<float>(p, st);
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

template <typename T>
static cudaError_t launch_logprobs_bwd(const BwdArgs& p, cudaStream_t st) {
    constexpr int stretch = LP_BWD_UNROLL * LP_BWD_THREADS * Vec<T>::N;             // (a row's vectors and its ends are not more than its length / N and one stretch)
    const dim3 grid((unsigned)p.T, (unsigned)((p.V + stretch - 1) / stretch));
    const bool together = ((reinterpret_cast<uintptr_t>(p.logits) ^ reinterpret_cast<uintptr_t>(p.dlogits)) & 15u) == 0 &&
                          (p.T == 1 || ((p.stride - p.grad_stride) * (long long)sizeof(T)) % 16 == 0);
    if (!together) return launch_pdl(logprobs_bwd_scalar_kernel<T>, grid, dim3(LP_BWD_THREADS), 0, st, 1, p);
    if (p.d_entropy != nullptr) return launch_pdl(logprobs_bwd_kernel<T, true>, grid, dim3(LP_BWD_THREADS), 0, st, 1, p);
    return launch_pdl(logprobs_bwd_kernel<T, false>, grid, dim3(LP_BWD_THREADS), 0, st, 1, p);
}

int launch_token_logprobs_bwd(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, const float* stats,
                              const float* d_logprobs, const float* d_entropy, long long grad_stride, void* dlogits, cudaStream_t st) {
    const BwdArgs p{T, V, row_stride, grad_stride, logits, tokens, c, stats, d_logprobs, d_entropy, dlogits};
    const cudaError_t err = dtype == QLORA_BF16 ? launch_logprobs_bwd<__nv_bfloat16>(p, st) : dtype == QLORA_FP16 ? launch_logprobs_bwd<__half>(p, st) : launch_logprobs_bwd<float>(p, st);
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

}  // namespace qlora
