// The optimizer step of the trainable pairs (Section 3.2, Eq. 3 of the paper: theta_l is optimised, theta_q stays): the global norm of
// all gradients, and AdamW over every tensor of a model in one launch, with 32-bit or 8-bit states.
#include <cuda_fp8.h>

#include <math.h>

#include "common.cuh"
#include "device_state.h"
#include "launch.h"

namespace qlora {

constexpr int OP_BLOCK = 256;            // elements that share one scale of the 8-bit states
constexpr int OP_THREADS = 256;
constexpr int OP_TABLE = 448;            // tensors per launch: their table travels in the kernel's parameters (32764 bytes at most)
constexpr int OP_PARTIALS = QLORA_GRAD_NORM_WORKSPACE_BYTES / sizeof(double);

// The tensors of one launch, cut into chunks of `chunk` elements (the last one of a tensor may be shorter): chunk c belongs to the tensor
// j with first[j] <= c < first[j + 1].
struct OptTable {
    qlora_adamw_tensor t[OP_TABLE];
    uint32_t first[OP_TABLE + 1];
    int n, chunk;
};

struct AdamScalars {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, weight_decay;
    float log_beta1, log_beta2;          // for a step number that is in device memory
    float lr, corr1, corr2;              // the rate, 1 - beta1^step, 1 - beta2^step
    int step;
    const float* lr_dev;
    const int32_t* step_dev;
    const float* norm;
};

__device__ __forceinline__ int tensor_of_chunk(const OptTable& tab, uint32_t c) {
    int lo = 0, hi = tab.n;              // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab.first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float e4m3_to_f(uint8_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
}

// Two numbers in [0, 2^20) from an element's place in its tensor and the number of the step.
__device__ __forceinline__ uint2 dither_of(uint32_t place, uint32_t step) {
    uint32_t x = place * 0x9E3779B1u + step * 0x7F4A7C15u;
    x = (x ^ (x >> 15)) * 0x2C1B3C6Du;
    x = (x ^ (x >> 13)) * 0x297A2D39u;
    x ^= x >> 16;
    return make_uint2(x >> 12, (x * 0x9E3779B1u) >> 12);
}

// x (at most 448 in size) to an e4m3 value beside it: adding the dither below the third fraction bit and cutting there goes up with a
// chance of the cut part's share of a step.  Below 2^-6 the steps stay 2^-9, those of the binade that x + 2^-6 lies in.
__device__ __forceinline__ float dithered_e4m3(float x, uint32_t dither) {
    const float a = fabsf(x), off = a < 0x1p-6f ? 0x1p-6f : 0.f;
    const float y = __uint_as_float((__float_as_uint(a + off) + dither) & 0xFFF00000u) - off;
    return copysignf(fminf(y, 448.f), x);
}

// One warp per 256 elements (8 per lane).
template <typename P, typename G, bool EIGHT>
__global__ void __launch_bounds__(OP_THREADS) adamw_kernel(const __grid_constant__ OptTable tab, const __grid_constant__ AdamScalars sc) {
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = tensor_of_chunk(tab, blockIdx.x);
    const qlora_adamw_tensor& t = tab.t[j];
    const long long begin = (long long)(blockIdx.x - tab.first[j]) * tab.chunk;
    const long long end = begin + tab.chunk < t.n ? begin + tab.chunk : t.n;
    const float f = sc.norm != nullptr ? sc.norm[1] : 1.f;
    if (!(fabsf(f) <= 3.402823466e38f)) return;
    const float lr = sc.lr_dev != nullptr ? *sc.lr_dev : sc.lr;
    int step = sc.step;
    float corr1 = sc.corr1, corr2 = sc.corr2;
    if (sc.step_dev != nullptr) {
        step = *sc.step_dev;
        corr1 = -expm1f((float)step * sc.log_beta1);
        corr2 = -expm1f((float)step * sc.log_beta2);
    }
    for (long long base = begin + warp * OP_BLOCK; base < end; base += OP_THREADS / 32 * OP_BLOCK) {
        float m[8], v[8];
        float ms = 0.f, us = 0.f;
        if (EIGHT) { ms = t.m_scale[base / OP_BLOCK]; us = t.v_scale[base / OP_BLOCK]; }
        float top_m = 0.f, top_u = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long e = base + i * 32 + lane;
            m[i] = v[i] = 0.f;
            if (e >= end) continue;
            const float g = f * to_f(static_cast<const G*>(t.grad)[e]);
            if (EIGHT) {
                m[i] = ms * e4m3_to_f(static_cast<const uint8_t*>(t.m)[e]);
                const float u = us * e4m3_to_f(static_cast<const uint8_t*>(t.v)[e]);
                v[i] = u * u;
            } else {
                m[i] = static_cast<const float*>(t.m)[e];
                v[i] = static_cast<const float*>(t.v)[e];
            }
            m[i] = sc.beta1 * m[i] + sc.one_minus_beta1 * g;
            v[i] = sc.beta2 * v[i] + sc.one_minus_beta2 * (g * g);
            float w = t.master != nullptr ? t.master[e] : to_f(static_cast<const P*>(t.param)[e]);
            w = w * (1.f - lr * sc.weight_decay) - lr * ((m[i] / corr1) / (sqrtf(v[i] / corr2) + sc.eps));
            if (t.master != nullptr) t.master[e] = w;
            static_cast<P*>(t.param)[e] = from_f<P>(w);
            if (EIGHT) {
                v[i] = sqrtf(v[i]);
                top_m = fmaxf(top_m, fabsf(m[i]));
                top_u = fmaxf(top_u, v[i]);
            } else {
                static_cast<float*>(t.m)[e] = m[i];
                static_cast<float*>(t.v)[e] = v[i];
            }
        }
        if (EIGHT) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                top_m = fmaxf(top_m, __shfl_xor_sync(0xFFFFFFFFu, top_m, o));
                top_u = fmaxf(top_u, __shfl_xor_sync(0xFFFFFFFFu, top_u, o));
            }
            const float im = top_m > 0x1p-100f ? 448.f / top_m : 0.f, iu = top_u > 0x1p-100f ? 448.f / top_u : 0.f;
            if (lane == 0) {
                t.m_scale[base / OP_BLOCK] = top_m > 0x1p-100f ? top_m * (1.f / 448.f) : 0.f;
                t.v_scale[base / OP_BLOCK] = top_u > 0x1p-100f ? top_u * (1.f / 448.f) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long e = base + i * 32 + lane;
                if (e >= end) continue;
                const uint2 r = dither_of((uint32_t)e, (uint32_t)step);
                const float cm = dithered_e4m3(m[i] * im, r.x), xu = v[i] * iu;
                float cu = dithered_e4m3(xu, r.y);
                if (xu > 0.f) cu = fmaxf(cu, 0x1p-9f);
                static_cast<uint8_t*>(t.m)[e] = __nv_cvt_float_to_fp8(cm, __NV_SATFINITE, __NV_E4M3);
                static_cast<uint8_t*>(t.v)[e] = __nv_cvt_float_to_fp8(cu, __NV_SATFINITE, __NV_E4M3);
            }
        }
    }
}

__device__ __forceinline__ double block_sum(double v) {           // the sum in thread 0, in a fixed order
    __shared__ double part[OP_THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        v = 0.0;
        for (int w = 0; w < OP_THREADS / 32; ++w) v += part[w];
    }
    return v;
}

// Sums of squares, one per block of the launch; `add`: on top of the previous launch's (more tensors than one table holds).
template <typename G>
__global__ void __launch_bounds__(OP_THREADS) grad_square_kernel(const __grid_constant__ OptTable tab, float prescale, int add, double* __restrict__ partial) {
    pdl_launch_dependents();
    pdl_wait();
    double acc = 0.0;
    for (uint32_t c = blockIdx.x; c < tab.first[tab.n]; c += gridDim.x) {
        const int j = tensor_of_chunk(tab, c);
        const qlora_adamw_tensor& t = tab.t[j];
        const long long begin = (long long)(c - tab.first[j]) * tab.chunk;
        const long long end = begin + tab.chunk < t.n ? begin + tab.chunk : t.n;
        const G* g = static_cast<const G*>(t.grad);
        for (long long e = begin + threadIdx.x; e < end; e += OP_THREADS) {
            const double x = (double)to_f(g[e]) * (double)prescale;
            acc = fma(x, x, acc);
        }
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + acc : acc;
}

__global__ void __launch_bounds__(OP_THREADS) grad_norm_kernel(int n, const double* __restrict__ partial, float prescale, float max_norm, float* __restrict__ out) {
    pdl_launch_dependents();
    pdl_wait();
    double acc = 0.0;
    for (int i = threadIdx.x; i < n; i += OP_THREADS) acc += partial[i];
    acc = block_sum(acc);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(acc);
        out[0] = norm;
        float f = prescale;
        if (max_norm > 0.f && norm > max_norm) f = prescale * (max_norm / norm);
        if (!(norm <= 3.402823466e38f)) f = __int_as_float(0x7FC00000);
        out[1] = f;
    }
}

// Fills the table with tensors from *at on; returns the number of chunks (0: nothing left).
static uint32_t fill_table(const qlora_adamw_desc& d, int* at, int chunk, OptTable& tab) {
    uint32_t chunks = 0;
    tab.n = 0;
    tab.chunk = chunk;
    while (*at < d.n_tensors && tab.n < OP_TABLE) {
        const qlora_adamw_tensor& t = d.tensors[*at];
        const uint32_t c = (uint32_t)((t.n + chunk - 1) / chunk);
        if (chunks > 0 && chunks + c > 0x7FFFFFFFu) break;
        if (c > 0) {
            tab.t[tab.n] = t;
            tab.first[tab.n++] = chunks;
            chunks += c;
        }
        ++*at;
    }
    tab.first[tab.n] = chunks;
    return chunks;
}

static int chunk_of(const qlora_adamw_desc& d) {
    (void)d;
    return 2048;
}

int launch_grad_norm(const qlora_adamw_desc& d, float prescale, float max_norm, float* out, void* workspace, cudaStream_t st) {
    static thread_local OptTable tab;
    double* partial = static_cast<double*>(workspace);
    int at = 0, used = 0;
    for (int launch = 0;; ++launch) {
        const uint32_t chunks = fill_table(d, &at, chunk_of(d), tab);
        if (chunks == 0) break;
        // (every launch on the grid of the first, whose partial sums the later ones add to)
        if (launch == 0) used = (int)(chunks < (uint32_t)OP_PARTIALS ? chunks : (uint32_t)OP_PARTIALS);
        cudaError_t err;
        if (d.grad_type == QLORA_FP32) err = launch_pdl(grad_square_kernel<float>, dim3(used), dim3(OP_THREADS), 0, st, 1, tab, prescale, launch, partial);
        else if (d.grad_type == QLORA_BF16) err = launch_pdl(grad_square_kernel<__nv_bfloat16>, dim3(used), dim3(OP_THREADS), 0, st, 1, tab, prescale, launch, partial);
        else err = launch_pdl(grad_square_kernel<__half>, dim3(used), dim3(OP_THREADS), 0, st, 1, tab, prescale, launch, partial);
        if (err != cudaSuccess) return QLORA_ERR_CUDA;
    }
    return launch_pdl(grad_norm_kernel, dim3(1), dim3(OP_THREADS), 0, st, 1, used, partial, prescale, max_norm, out) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

template <typename P, typename G>
static cudaError_t launch_adamw_as(bool eight, uint32_t chunks, const OptTable& tab, const AdamScalars& sc, cudaStream_t st) {
    if (eight) return launch_pdl(adamw_kernel<P, G, true>, dim3(chunks), dim3(OP_THREADS), 0, st, 1, tab, sc);
    return launch_pdl(adamw_kernel<P, G, false>, dim3(chunks), dim3(OP_THREADS), 0, st, 1, tab, sc);
}

template <typename P>
static cudaError_t launch_adamw_param(int grad_type, bool eight, uint32_t chunks, const OptTable& tab, const AdamScalars& sc, cudaStream_t st) {
    if (grad_type == QLORA_FP32) return launch_adamw_as<P, float>(eight, chunks, tab, sc, st);
    if (grad_type == QLORA_BF16) return launch_adamw_as<P, __nv_bfloat16>(eight, chunks, tab, sc, st);
    return launch_adamw_as<P, __half>(eight, chunks, tab, sc, st);
}

int launch_adamw(const qlora_adamw_desc& d, double lr, int step, const float* lr_dev, const int32_t* step_dev, const float* norm, cudaStream_t st) {
    static thread_local OptTable tab;
    AdamScalars sc;
    sc.beta1 = (float)d.beta1; sc.one_minus_beta1 = (float)(1.0 - d.beta1);
    sc.beta2 = (float)d.beta2; sc.one_minus_beta2 = (float)(1.0 - d.beta2);
    sc.eps = (float)d.eps; sc.weight_decay = (float)d.weight_decay;
    sc.log_beta1 = (float)log(d.beta1); sc.log_beta2 = (float)log(d.beta2);
    sc.lr = (float)lr;
    sc.corr1 = (float)-expm1(step * log(d.beta1)); sc.corr2 = (float)-expm1(step * log(d.beta2));
    sc.step = step; sc.lr_dev = lr_dev; sc.step_dev = step_dev; sc.norm = norm;
    int at = 0;
    for (;;) {
        const uint32_t chunks = fill_table(d, &at, chunk_of(d), tab);
        if (chunks == 0) return QLORA_OK;
        cudaError_t err;
        const bool eight = d.state_type == QLORA_E4M3;
        if (d.param_type == QLORA_BF16) err = launch_adamw_param<__nv_bfloat16>(d.grad_type, eight, chunks, tab, sc, st);
        else if (d.param_type == QLORA_FP16) err = launch_adamw_param<__half>(d.grad_type, eight, chunks, tab, sc, st);
        else err = launch_adamw_param<float>(d.grad_type, eight, chunks, tab, sc, st);
        if (err != cudaSuccess) return QLORA_ERR_CUDA;
    }
}

}  // namespace qlora
