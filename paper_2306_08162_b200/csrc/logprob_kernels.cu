// Log probabilities of given tokens over [T, V] logits, with each row's entropy and most likely alternatives, and their gradient with
// respect to the logits.  Per row, with c the inverse temperature, m = max z and d_j = c (z_j - m) <= 0:
//     s = sum exp d_j,    log p_j = d_j - log s,    H = log s - (sum exp(d_j) d_j) / s
// in one pass over the row: every thread keeps its own maximum and sums relative to it and corrects them when the maximum moves.
#include "common.cuh"
#include "device_state.h"
#include "launch.h"

namespace qlora {

constexpr int LP_THREADS = 256;

__device__ __forceinline__ float lp_f(float x) { return x; }
__device__ __forceinline__ float lp_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float lp_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T lp_to(float x);
template <> __device__ __forceinline__ float lp_to<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 lp_to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half lp_to<__half>(float x) { return __float2half_rn(x); }

// The order of the alternatives: larger logits first (a NaN before all, -0 with 0), equal ones by their place.  Larger keys come first.
__device__ __forceinline__ uint32_t order_key(float z) {
    if (z != z) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t entry_key(float z, int j) { return (uint64_t)order_key(z) << 32 | (uint32_t)~j; }

// Running maximum and sums relative to it.
struct RowSums {
    float m, s, a;                       // a = sum exp(d) d
};
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Moves the sums to a maximum m >= x.m.
__device__ __forceinline__ void rebase(RowSums& x, float m, float c) {
    const float d = fmaxf((x.m - m) * c, -1e30f);                 // (nothing yet: x.m = -inf, and maybe m too: NaN becomes -1e30)
    const float e = expf(d);
    x.a = e * fmaf(x.s, d, x.a);
    x.s *= e;
    x.m = m;
}
__device__ __forceinline__ RowSums merged(RowSums x, RowSums y, float c) {
    const float m = max_nan(x.m, y.m);
    rebase(x, m, c);
    rebase(y, m, c);
    return RowSums{m, x.s + y.s, x.a + y.a};
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
    const T* z = logits + row * stride;
    RowSums x{-INFINITY, 0.f, 0.f};
    for (int j = threadIdx.x; j < V; j += LP_THREADS) x = merged(x, RowSums{lp_f(z[j]), 1.f, 0.f}, c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        x = merged(x, RowSums{__shfl_xor_sync(0xFFFFFFFFu, x.m, o), __shfl_xor_sync(0xFFFFFFFFu, x.s, o), __shfl_xor_sync(0xFFFFFFFFu, x.a, o)}, c);
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    x = sums[0];
    for (int w = 1; w < LP_THREADS / 32; ++w) x = merged(x, sums[w], c);
    const bool none = x.m == -INFINITY, bad = !(x.m < INFINITY);
    float logs = logf(x.s), H = fmaxf(logs - x.a / x.s, 0.f);
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
