// Log probabilities of given tokens over [T, V] logits, with each row's entropy and most likely alternatives, and their gradient with
// respect to the logits.  Per row, with c the inverse temperature, m = max z and d_j = c (z_j - m) <= 0:
//     s = sum exp d_j,    log p_j = d_j - log s,    H = log s - (sum exp(d_j) d_j) / s
// in one pass over the row: every thread keeps its own maximum and sums relative to it and corrects them when the maximum moves.
#include "common.cuh"
#include "device_state.h"
#include "f32x2.cuh"
#include "launch.h"

namespace qlora {

constexpr int LP_THREADS = 512;
constexpr int LP_UNROLL = 4;             // 16-byte vectors that a thread has on their way at a time
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
    int head, vectors, tail;             // tail: where the rest begins
    __device__ __forceinline__ RowParts(const T* row, int V) : z(row) {
        head = min(V, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(row)) & 15u) / (int)sizeof(T));
        vectors = (V - head) / Vec<T>::N;
        tail = head + vectors * Vec<T>::N;
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
__device__ __forceinline__ uint64_t entry_key(float z, int j) { return (uint64_t)order_key(z) << 32 | (uint32_t)~j; }

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
template <typename T>
__device__ __forceinline__ RowSums thread_sums(const RowParts<T>& row, int V, float kd) {
    RowSums x{-INFINITY, 0.f, 0.f};
    const f2 kd2 = make_f2(kd, kd);
    const uint4* body = row.body();
    for (int c0 = threadIdx.x; c0 < row.vectors; c0 += LP_UNROLL * LP_THREADS) {
        uint4 v[LP_UNROLL];
        typename Vec<T>::Max top = Vec<T>::lowest();
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * LP_THREADS < row.vectors) v[u] = load_stream(body + c0 + u * LP_THREADS);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * LP_THREADS < row.vectors) top = Vec<T>::fold(top, v[u]);
        const float m = max_nan(x.m, Vec<T>::value(top));
        if (m != x.m) rebase(x, m, kd);
        const f2 minus_m = make_f2(-m, -m);
        f2 s2 = make_f2(x.s, 0.f), a2 = make_f2(x.a, 0.f);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
            if (c0 + u * LP_THREADS < row.vectors) {
#pragma unroll
                for (int i = 0; i < Vec<T>::N / 2; ++i) add_pair(s2, a2, Vec<T>::pair(v[u], i), minus_m, kd2);
            }
        x.s = lo_of(s2) + hi_of(s2);
        x.a = lo_of(a2) + hi_of(a2);
    }
    if ((int)threadIdx.x < row.head) add_one(x, lp_f(row.z[threadIdx.x]), kd);
    if (row.tail + (int)threadIdx.x < V) add_one(x, lp_f(row.z[row.tail + threadIdx.x]), kd);
    return x;
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(int V, long long stride, const T* __restrict__ logits, const int32_t* __restrict__ tokens, float c, int k,
                                                              float* __restrict__ logprobs, float* __restrict__ entropy, int32_t* __restrict__ top_ids,
                                                              float* __restrict__ top_logprobs, float* __restrict__ stats) {
    __shared__ RowSums sums[LP_THREADS / 32];
    __shared__ uint64_t best[LP_THREADS / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float kd = c * kLog2e;
    const T* z = logits + row * stride;
    const RowParts<T> parts(z, V);
    RowSums x = warp_merge(thread_sums(parts, V, kd), kd);
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    x = warp_merge(lane < LP_THREADS / 32 ? sums[lane] : RowSums{-INFINITY, 0.f, 0.f}, kd);
    const bool none = x.m == -INFINITY, bad = !(x.m < INFINITY);
    float logs = logf(x.s), H = fmaxf(logs - c * (x.a / x.s), 0.f);
    if (none) { logs = -INFINITY; H = 0.f; }
    if (bad) x.m = logs = H = __int_as_float(0x7FC00000);
    auto logp = [&](float zj) { return none ? -INFINITY : (zj - x.m) * c - logs; };
    if (threadIdx.x == 0) {
        if (stats != nullptr) { stats[3ll * row] = x.m; stats[3ll * row + 1] = logs; stats[3ll * row + 2] = H; }
        if (entropy != nullptr) entropy[row] = H;
        if (logprobs != nullptr) {
            const int t = tokens[row];
            logprobs[row] = t >= 0 && t < V ? logp(lp_f(z[t])) : 0.f;
        }
    }
    uint64_t last = ~0ull;
    for (int i = 0; i < k; ++i) {                                  // the largest entry below the one before
        uint64_t b = 0;
        for (int j = threadIdx.x; j < V; j += LP_THREADS) {
            const uint64_t e = entry_key(lp_f(z[j]), j);
            if ((e < last || i == 0) && e > b) b = e;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor_sync(0xFFFFFFFFu, b, o);
            if (other > b) b = other;
        }
        __syncthreads();
        if (lane == 0) best[warp] = b;
        __syncthreads();
        for (int w = 0; w < LP_THREADS / 32; ++w)
            if (best[w] > b) b = best[w];
        last = b;
        if (threadIdx.x == 0) {
            const int j = (int)~(uint32_t)last;
            if (top_ids != nullptr) top_ids[(long long)row * k + i] = j;
            if (top_logprobs != nullptr) top_logprobs[(long long)row * k + i] = logp(lp_f(z[j]));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_bwd_kernel(int V, long long stride, const T* logits, const int32_t* __restrict__ tokens, float c,
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
    for (int j = threadIdx.x; j < V; j += LP_THREADS) {
        float g = 0.f;
        if (!zero) {
            const float lp = (lp_f(z[j]) - m) * c - logs, p = expf(lp);
            g = -p * (gl + gh * (fmaxf(lp, -1e30f) + H)) + (j == t ? gl : 0.f);
            if (m != m) g = m;
        }
        dz[j] = lp_to<T>(g);
    }
}

int launch_token_logprobs(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, int k, float* logprobs,
                          float* entropy, int32_t* top_ids, float* top_logprobs, float* stats, cudaStream_t st) {
    cudaError_t err;
#define QLORA_LP(TYPE)                                                                                                                              \
    err = launch_pdl(logprobs_kernel<TYPE>, dim3((unsigned)T), dim3(LP_THREADS), 0, st, 1, V, row_stride, (const TYPE*)logits, tokens, c, k, logprobs, \
                     entropy, top_ids, top_logprobs, stats)
    if (dtype == QLORA_BF16) QLORA_LP(__nv_bfloat16);
    else if (dtype == QLORA_FP16) QLORA_LP(__half);
    else QLORA_LP(float);
#undef QLORA_LP
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

int launch_token_logprobs_bwd(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens, float c, const float* stats,
                              const float* d_logprobs, const float* d_entropy, long long grad_stride, void* dlogits, cudaStream_t st) {
    cudaError_t err;
#define QLORA_LP(TYPE)                                                                                                                              \
    err = launch_pdl(logprobs_bwd_kernel<TYPE>, dim3((unsigned)T), dim3(LP_THREADS), 0, st, 1, V, row_stride, (const TYPE*)logits, tokens, c, stats,  \
                     d_logprobs, d_entropy, grad_stride, (TYPE*)dlogits)
    if (dtype == QLORA_BF16) QLORA_LP(__nv_bfloat16);
    else if (dtype == QLORA_FP16) QLORA_LP(__half);
    else QLORA_LP(float);
#undef QLORA_LP
    return err == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

}  // namespace qlora
