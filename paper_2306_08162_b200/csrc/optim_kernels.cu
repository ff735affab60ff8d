// The optimizer step of the trainable pairs (Section 3.2, Eq. 3 of the paper: theta_l is optimised, theta_q stays): the global norm of
// all gradients, and AdamW over every tensor of a model in one launch, with 32-bit or 8-bit states.
// 32-bit states: bound by HBM.  Rank 32 on all projections of 32 layers (80 M elements in 448 tensors, bf16 weights, 24 bytes an element): 277 us, 6.9 TB/s;
// rank 64 with fp32 master weights behind the norm: 803 us, where the step's bytes alone take 734 at the copy rate and the gradients' second reading 98.
// 8-bit states: the same 80 M elements in 177 us, 5.4 TB/s, 234 us behind the norm, where their bytes take 147.  No unit is full: 58 instructions an element are 130 us
// of issue, which is 74 % busy, two fifths of them on the integer pipe (some 60 %), DRAM 57 %; 62 registers a thread leave 43 % of the warps to cover the latencies.
// Rate and step number from device memory stand ahead of the loads: 192 us.
// A block of threads has one chunk, 8 elements a thread, and ends: with more of them in a loop (2 to 8, with or without the next one's loads ahead) the
// blocks of an SM load and compute in step with each other, 190 to 290 us.
#include <cuda_fp8.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "device_state.h"
#include "f32x2.cuh"
#include "launch.h"

namespace qlora {

constexpr int OP_BLOCK = 256;            // elements that share one scale of the 8-bit states, and that a warp handles at a time
constexpr int OP_THREADS = 256;
constexpr int OP_CHUNK = 2048;           // elements of a chunk: a block of 256 to each of 8 warps
// Tensors per launch: their table travels in the kernel's parameters (32764 bytes at most), and a launch costs the host more the larger it is.
constexpr int OP_TABLE = 448, OP_MIDDLE_TABLE = 128, OP_SMALL_TABLE = 16;
constexpr int OP_CLUSTER = 8, OP_CLUSTER_CHUNKS = 64;
constexpr int OP_PARTIALS = QLORA_GRAD_NORM_WORKSPACE_BYTES / sizeof(double);

// The tensors of one launch, cut into chunks of OP_CHUNK elements (the last one of a tensor may be shorter): chunk c belongs to the tensor
// j with first[j] <= c < first[j + 1], which is near[c >> near_log2] or one of the next.
template <int CAP>
struct OptTable {
    qlora_adamw_tensor t[CAP];
    uint32_t first[CAP + 1];
    int n, near_log2;
    uint16_t near[CAP];
};
static_assert(sizeof(OptTable<OP_TABLE>) <= 32000, "a kernel's parameters");

struct AdamScalars {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, weight_decay;
    float log_beta1, log_beta2;          // for a step number that is in device memory
    float lr, inv_corr1, root_inv_corr2; // the rate, 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    int step;
    const float* lr_dev;
    const int32_t* step_dev;
    const float* norm;
};

template <int CAP>
__device__ __forceinline__ int tensor_of_chunk(const OptTable<CAP>& tab, uint32_t c) {
    int j = tab.near[c >> tab.near_log2];
    while (tab.first[j + 1] <= c) ++j;                               // (c is below first[n])
    return j;
}

// Two numbers below 2^32 from an element's place in its tensor and the number of the step (x: place * 0x9E3779B1 + step * 0x7F4A7C15); the
// dither of a code is the upper 20 bits.
__device__ __forceinline__ uint2 dither_of(uint32_t x) {
    x = (x ^ (x >> 15)) * 0x2C1B3C6Du;
    x = (x ^ (x >> 13)) * 0x297A2D39u;
    x ^= x >> 16;
    return make_uint2(x, x * 0x9E3779B1u);
}

// The e4m3 code beside y 2^120, y >= 0, in the top byte of the result: times 2^-120 the values that e4m3 holds, its smallest ones with fewer than three
// fraction bits among them, are fp32's own with the same exponents and fractions, 20 bits further up.  Adding the dither below the code and cutting
// there goes up with a chance of the cut part's share of a step.  (y's sign and the dither's lower bits fall out at the ends.)
__device__ __forceinline__ uint32_t dithered_code(uint32_t y, uint32_t dither) { return y * 16u + (dither >> 8); }
// Bytes 3 of four words.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// Four codes without a sign: 0x7F to 0x7E, the code of 448 (the rounding of 448 / top can put the top one just above).
__device__ __forceinline__ uint32_t at_most_448(uint32_t codes) { return codes - (((codes + 0x01010101u) >> 7) & 0x01010101u); }

// Four consecutive elements (of 16-byte aligned tensors, at a multiple of 4).
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y));
}
__device__ __forceinline__ float4 load4(const __half* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 load4(const uint8_t* p) {             // e4m3
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    const __half2 a = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xFFFFu), __NV_E4M3));
    const __half2 b = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> 16), __NV_E4M3));
    const float2 x = __half22float2(a), y = __half22float2(b);
    return make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void store4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store4(__half* p, const float* v) {
    const __half2 a = __floats2half2_rn(v[0], v[1]), b = __floats2half2_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float one(const float* p) { return *p; }
__device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float one(const uint8_t* p) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(*p, __NV_E4M3))); }
__device__ __forceinline__ void put_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put_one(__half* p, float v) { *p = __float2half_rn(v); }

// This lane's 8 of a block of 256 elements: 4 at 4 lane and 4 at 128 + 4 lane, so that every access of a warp is contiguous.  `left`: elements of
// the block that are there; FULL: all 256 (all but the last block of a tensor).
template <bool FULL, typename E>
__device__ __forceinline__ void load8(const E* p, uint32_t base, uint32_t lane, int left, float (&v)[8]) {
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t in = 128 * h + 4 * lane, at = base + in;
        if (FULL || (int)in + 4 <= left) {
            const float4 x = load4(p + at);
            v[4 * h] = x.x; v[4 * h + 1] = x.y; v[4 * h + 2] = x.z; v[4 * h + 3] = x.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = (int)in + i < left ? one(p + at + i) : 0.f;
        }
    }
}
template <bool FULL, typename E>
__device__ __forceinline__ void store8(E* p, uint32_t base, uint32_t lane, int left, const float (&v)[8]) {
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t in = 128 * h + 4 * lane, at = base + in;
        if (FULL || (int)in + 4 <= left) store4(p + at, v + 4 * h);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((int)in + i < left) put_one(p + at + i, v[4 * h + i]);
    }
}

// (The errors of this root and of the update's quotient are 2^-22 of an update that is a small part of its weight.  Not the form that takes numbers below
// 2^-126 for zero: a second moment there has a root of up to 2^-63, far above the smallest eps.  In the 8-bit step that costs 1.2 % of its time.)
__device__ __forceinline__ float fast_sqrt(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The largest of a warp's values from 0 on (their bits are in order; a NaN is above all).
__device__ __forceinline__ float warp_top(float lane_top) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(lane_top))); }
__device__ __forceinline__ void fold_top(float& top, f2 x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(lo_of(x))));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(hi_of(x))));
}
__device__ __forceinline__ f2 both(float x) { return make_f2(x, x); }
__device__ __forceinline__ float inverse_ftz(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The step of a block with 8-bit states.  Instructions are most of its time, so arithmetic goes by pairs and one square root serves the update and the state.
struct AdamBlock {                                                   // what holds for the whole call
    float f, minus_decay, rate, root_inv2;                           // -lr weight_decay (1 - lr weight_decay, rounded, would be off by up to half of 2^-24 at every step)
    uint32_t step_term;
};
// The tensors from the chunk's first element on.  (The same for the whole block; a thread adds 32 bits to them.)
template <typename P, typename G, typename S>
struct Chunk {
    P* param;
    float* master;
    const G* grad;
    S *m, *v;
    float *m_scale, *v_scale;
    uint32_t place;                                                  // of its first element in the tensor
    __device__ __forceinline__ Chunk(const qlora_adamw_tensor& t, long long begin)
        : param(static_cast<P*>(t.param) + begin), master(t.master != nullptr ? t.master + begin : nullptr), grad(static_cast<const G*>(t.grad) + begin),
          m(static_cast<S*>(t.m) + begin), v(static_cast<S*>(t.v) + begin), m_scale(t.m_scale + begin / OP_BLOCK), v_scale(t.v_scale + begin / OP_BLOCK), place((uint32_t)begin) {}
};

template <typename P, typename G, bool FULL>
__device__ __forceinline__ void adamw8_block(const Chunk<P, G, uint8_t>& t, const AdamScalars& sc, const AdamBlock& k, uint32_t base, int left, uint32_t lane) {
    float g[8], w[8], mc[8], uc[8];
    load8<FULL>(t.grad, base, lane, left, g);
    load8<FULL>(t.m, base, lane, left, mc);
    load8<FULL>(t.v, base, lane, left, uc);
    if (t.master != nullptr) load8<FULL>(t.master, base, lane, left, w);
    else load8<FULL>(t.param, base, lane, left, w);
    const float ms = t.m_scale[base / OP_BLOCK], us = t.v_scale[base / OP_BLOCK];
    const f2 m_by = both(sc.beta1 * ms), one_minus1 = both(sc.one_minus_beta1), u_by = both(us), beta2 = both(sc.beta2), one_minus2 = both(sc.one_minus_beta2);
    f2 m[4], u[4];
    float top_m = 0.f, top_u = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f2 gi = mul2(make_f2(g[2 * i], g[2 * i + 1]), both(k.f));
        m[i] = fma2(make_f2(mc[2 * i], mc[2 * i + 1]), m_by, mul2(gi, one_minus1));
        const f2 old = mul2(make_f2(uc[2 * i], uc[2 * i + 1]), u_by);
        const f2 v = fma2(mul2(old, old), beta2, mul2(mul2(gi, gi), one_minus2));
        u[i] = make_f2(fast_sqrt(lo_of(v)), fast_sqrt(hi_of(v)));
        const f2 den = fma2(u[i], both(k.root_inv2), both(sc.eps));
        const f2 q = mul2(mul2(m[i], both(-k.rate)), make_f2(inverse_ftz(lo_of(den)), inverse_ftz(hi_of(den))));
        const f2 old_w = make_f2(w[2 * i], w[2 * i + 1]), wi = add2(old_w, fma2(old_w, both(k.minus_decay), q));
        w[2 * i] = lo_of(wi);
        w[2 * i + 1] = hi_of(wi);
        fold_top(top_m, m[i]);
        fold_top(top_u, u[i]);
    }
    if (t.master != nullptr) store8<FULL>(t.master, base, lane, left, w);
    store8<FULL>(t.param, base, lane, left, w);
    top_m = warp_top(top_m);
    top_u = warp_top(top_u);
    const bool held_m = !(top_m <= 0x1p-100f), held_u = !(top_u <= 0x1p-100f);
    const f2 inv_m = both(held_m ? 448.f * inverse_ftz(top_m) : 0.f), inv_u = both(held_u ? 448.f * inverse_ftz(top_u) : 0.f), down = both(0x1p-120f);
    const uint32_t place = (t.place + base + 4u * lane) * 0x9E3779B1u + k.step_term;
#pragma unroll
    for (int q = 0; q < 2; ++q) {                                    // four consecutive elements
        uint32_t cm[4], cu[4], sign[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 2 * q + e / 2;
            const f2 y = mul2(mul2(m[i], inv_m), down), r = mul2(mul2(u[i], inv_u), down);
            const uint2 d = dither_of(place + (128u * q + e) * 0x9E3779B1u);
            sign[e] = __float_as_uint(e & 1 ? hi_of(y) : lo_of(y));
            cm[e] = dithered_code(sign[e], d.x);
            // (a root above zero has a code above zero: its bits are far above 2^20, those of zero are not)
            const uint32_t least = min(__float_as_uint(e & 1 ? hi_of(u[i]) : lo_of(u[i])), 1u << 24);
            cu[e] = max(dithered_code(__float_as_uint(e & 1 ? hi_of(r) : lo_of(r)), d.y), least);
        }
        const uint32_t codes_m = at_most_448(top_bytes(cm[0], cm[1], cm[2], cm[3]) & 0x7F7F7F7Fu) | (top_bytes(sign[0], sign[1], sign[2], sign[3]) & 0x80808080u);
        const uint32_t codes_u = at_most_448(top_bytes(cu[0], cu[1], cu[2], cu[3]));
        const uint32_t in = 128 * q + 4 * lane, at = base + in;
        if (FULL || (int)in + 4 <= left) {
            *reinterpret_cast<uint32_t*>(t.m + at) = codes_m;
            *reinterpret_cast<uint32_t*>(t.v + at) = codes_u;
        } else {
            for (int e = 0; e < 4; ++e)
                if ((int)in + e < left) {
                    t.m[at + e] = (uint8_t)(codes_m >> (8 * e));
                    t.v[at + e] = (uint8_t)(codes_u >> (8 * e));
                }
        }
    }
    if (lane == 0) {
        t.m_scale[base / OP_BLOCK] = held_m ? top_m * (1.f / 448.f) : 0.f;
        t.v_scale[base / OP_BLOCK] = held_u ? top_u * (1.f / 448.f) : 0.f;
    }
}

template <typename P, typename G, bool FULL>
__device__ __forceinline__ void adamw32_block(const Chunk<P, G, float>& t, const AdamScalars& sc, const AdamBlock& k, uint32_t base, int left, uint32_t lane) {
    float g[8], w[8], m[8], v[8];
    load8<FULL>(t.grad, base, lane, left, g);
    if (t.master != nullptr) load8<FULL>(t.master, base, lane, left, w);
    else load8<FULL>(t.param, base, lane, left, w);
    load8<FULL>(t.m, base, lane, left, m);
    load8<FULL>(t.v, base, lane, left, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = k.f * g[i];
        m[i] = fmaf(sc.beta1, m[i], sc.one_minus_beta1 * gi);
        v[i] = fmaf(sc.beta2, v[i], sc.one_minus_beta2 * (gi * gi));
        w[i] += fmaf(w[i], k.minus_decay, -__fdividef(k.rate * m[i], fmaf(fast_sqrt(v[i]), k.root_inv2, sc.eps)));
    }
    if (t.master != nullptr) store8<FULL>(t.master, base, lane, left, w);
    store8<FULL>(t.param, base, lane, left, w);
    store8<FULL>(t.m, base, lane, left, m);
    store8<FULL>(t.v, base, lane, left, v);
}

// A chunk to a block of threads, 256 elements to a warp (8 per lane).
template <typename P, typename G, bool EIGHT, int CAP>
__global__ void __launch_bounds__(OP_THREADS, 4) adamw_kernel(const __grid_constant__ OptTable<CAP> tab, const __grid_constant__ AdamScalars sc) {
    __shared__ float corr[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    const int j = tensor_of_chunk(tab, blockIdx.x);
    const long long begin = (long long)(blockIdx.x - tab.first[j]) * OP_CHUNK;
    const Chunk<P, G, std::conditional_t<EIGHT, uint8_t, float>> t(tab.t[j], begin);
    const int n = (int)min((long long)OP_CHUNK, tab.t[j].n - begin);
    pdl_wait();
    const float f = sc.norm != nullptr ? sc.norm[1] : 1.f;
    const float lr = sc.lr_dev != nullptr ? *sc.lr_dev : sc.lr;
    const int step = sc.step_dev != nullptr ? *sc.step_dev : sc.step;
    float inv1 = sc.inv_corr1, root_inv2 = sc.root_inv_corr2;
    if (sc.step_dev != nullptr) {
        if (threadIdx.x == 0) {
            corr[0] = 1.f / -expm1f((float)step * sc.log_beta1);
            corr[1] = rsqrtf(-expm1f((float)step * sc.log_beta2));
        }
        __syncthreads();
        inv1 = corr[0];
        root_inv2 = corr[1];
    }
    if (!(fabsf(f) < INFINITY)) return;
    const AdamBlock k{f, -lr * sc.weight_decay, lr * inv1, root_inv2, (uint32_t)step * 0x7F4A7C15u};
    const uint32_t base = warp * OP_BLOCK;
    const int left = min(n - (int)base, OP_BLOCK);
    if constexpr (EIGHT) {
        if (n == OP_CHUNK) adamw8_block<P, G, true>(t, sc, k, base, left, lane);
        else if (left > 0) adamw8_block<P, G, false>(t, sc, k, base, left, lane);
    } else {
        if (n == OP_CHUNK) adamw32_block<P, G, true>(t, sc, k, base, left, lane);
        else if (left > 0) adamw32_block<P, G, false>(t, sc, k, base, left, lane);
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

__device__ __forceinline__ uint4 load_once(const uint4* p) {            // 16 bytes, not kept in L1 (asm volatile: several loads stay ahead of their uses)
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename G>
__device__ __forceinline__ void add_squares(double& acc, const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(G) == 4) {
            const double x = (double)__uint_as_float(w[i]);
            acc = fma(x, x, acc);
        } else {
            float2 f;
            if constexpr (std::is_same_v<G, __half>) f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            else f = make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
            acc = fma((double)f.x, (double)f.x, acc);
            acc = fma((double)f.y, (double)f.y, acc);
        }
    }
}

// The sum of squares of chunks c to stop - 1, this thread's part: in 64 bits, since a square can leave fp32's range and HBM leaves the time.
template <typename G, int CAP>
__device__ __forceinline__ double squares_of(const OptTable<CAP>& tab, int j, uint32_t c, uint32_t stop) {
    constexpr int PER = 16 / sizeof(G), UNROLL = 4;
    double acc = 0.0;
    for (; c < stop; ++j) {                                          // the stretch's part of one tensor after the other (c lies in tensor j)
        const qlora_adamw_tensor& t = tab.t[j];
        const uint32_t next = min(stop, tab.first[j + 1]);
        const long long begin = (long long)(c - tab.first[j]) * OP_CHUNK, end = min((long long)(next - tab.first[j]) * OP_CHUNK, t.n);
        const G* grad = static_cast<const G*>(t.grad) + begin;
        const long long vectors = (end - begin) / PER;
        const uint4* body = reinterpret_cast<const uint4*>(grad);
        long long at = threadIdx.x;
        for (; at + (UNROLL - 1) * OP_THREADS < vectors; at += UNROLL * OP_THREADS) {
            uint4 v[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = load_once(body + at + u * OP_THREADS);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) add_squares<G>(acc, v[u]);
        }
        for (; at < vectors; at += OP_THREADS) add_squares<G>(acc, load_once(body + at));
        for (long long e = vectors * PER + threadIdx.x; e < end - begin; e += OP_THREADS) acc = fma((double)one(grad + e), (double)one(grad + e), acc);
        c = next;
    }
    return acc;
}
__device__ __forceinline__ void tell_norm(double squares, float prescale, float max_norm, float* out) {
    const float norm = (float)(sqrt(squares) * fabs((double)prescale));
    float f = prescale;
    if (max_norm > 0.f && norm > max_norm) f = prescale * (max_norm / norm);
    if (!(norm < INFINITY)) f = __int_as_float(0x7FC00000);
    out[0] = norm;
    out[1] = f;
}

// One partial sum to each block of the launch, which has a stretch of the chunks (the same number to within one); `add`: on top of the
// previous launch's (more tensors than one table holds).
template <typename G, int CAP>
__global__ void __launch_bounds__(OP_THREADS) grad_square_kernel(const __grid_constant__ OptTable<CAP> tab, int add, double* __restrict__ partial) {
    pdl_launch_dependents();
    const uint64_t chunks = tab.first[tab.n];
    const uint32_t c = (uint32_t)(chunks * blockIdx.x / gridDim.x), stop = (uint32_t)(chunks * (blockIdx.x + 1) / gridDim.x);
    const int j = c < stop ? tensor_of_chunk(tab, c) : 0;
    pdl_wait();
    const double acc = block_sum(squares_of<G>(tab, j, c, stop));
    if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + acc : acc;
}

__global__ void __launch_bounds__(OP_THREADS) grad_norm_kernel(int n, const double* __restrict__ partial, float prescale, float max_norm, float* __restrict__ out) {
    pdl_launch_dependents();
    pdl_wait();
    double acc = 0.0;
    for (int i = threadIdx.x; i < n; i += OP_THREADS) acc += partial[i];
    acc = block_sum(acc);
    if (threadIdx.x == 0) tell_norm(acc, prescale, max_norm, out);
}

// Few chunks: all of it in one launch, a cluster of OP_CLUSTER blocks whose sums meet in the shared memory of the first.
template <typename G, int CAP>
__global__ void __launch_bounds__(OP_THREADS) grad_norm_cluster_kernel(const __grid_constant__ OptTable<CAP> tab, float prescale, float max_norm, float* __restrict__ out) {
    __shared__ double sums[OP_CLUSTER];
    pdl_launch_dependents();
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");    // this block has begun: the others may write to its shared memory
    const uint32_t chunks = tab.first[tab.n], c = chunks * blockIdx.x / OP_CLUSTER, stop = chunks * (blockIdx.x + 1) / OP_CLUSTER;
    const int j = c < stop ? tensor_of_chunk(tab, c) : 0;
    pdl_wait();
    double acc = block_sum(squares_of<G>(tab, j, c, stop));
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (threadIdx.x == 0) {
        uint32_t at;
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&sums[blockIdx.x])));
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(acc) : "memory");
    }
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        acc = 0.0;
        for (int b = 0; b < OP_CLUSTER; ++b) acc += sums[b];
        tell_norm(acc, prescale, max_norm, out);
    }
}

// Fills the table with tensors from *at on; returns the number of chunks (0: nothing left).
template <int CAP>
static uint32_t fill_table(const qlora_adamw_desc& d, int* at, OptTable<CAP>& tab) {
    uint32_t chunks = 0;
    tab.n = 0;
    while (*at < d.n_tensors && tab.n < CAP) {
        const qlora_adamw_tensor& t = d.tensors[*at];
        const uint32_t c = (uint32_t)((t.n + OP_CHUNK - 1) / OP_CHUNK);
        if (chunks > 0 && chunks + c > 0x7FFFFFFFu) break;
        if (c > 0) {
            tab.t[tab.n] = t;
            tab.first[tab.n++] = chunks;
            chunks += c;
        }
        ++*at;
    }
    tab.first[tab.n] = chunks;
    tab.near_log2 = 0;
    while (chunks > 0 && ((chunks - 1) >> tab.near_log2) >= (uint32_t)CAP) ++tab.near_log2;
    int j = 0;
    for (uint32_t i = 0; chunks > 0 && i <= (chunks - 1) >> tab.near_log2; ++i) {
        while (tab.first[j + 1] <= i << tab.near_log2) ++j;
        tab.near[i] = (uint16_t)j;
    }
    return chunks;
}

template <typename G, int CAP>
static int launch_grad_norm_as(const qlora_adamw_desc& d, float prescale, float max_norm, float* out, void* workspace, cudaStream_t st) {
    static thread_local OptTable<CAP> tab;
    double* partial = static_cast<double*>(workspace);
    const int most = 4 * sm_count() < OP_PARTIALS ? 4 * sm_count() : OP_PARTIALS;
    int at = 0, used = 0;
    for (int launch = 0;; ++launch) {
        const uint32_t chunks = fill_table(d, &at, tab);
        if (chunks == 0) break;
        if (launch == 0 && at == d.n_tensors && chunks <= OP_CLUSTER_CHUNKS)
            return launch_pdl(grad_norm_cluster_kernel<G, CAP>, dim3(OP_CLUSTER), dim3(OP_THREADS), 0, st, OP_CLUSTER, tab, prescale, max_norm, out) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
        // (every launch on the grid of the first, whose partial sums the later ones add to)
        if (launch == 0) used = (int)(chunks < (uint32_t)most ? chunks : (uint32_t)most);
        if (launch_pdl(grad_square_kernel<G, CAP>, dim3(used), dim3(OP_THREADS), 0, st, 1, tab, launch, partial) != cudaSuccess) return QLORA_ERR_CUDA;
    }
    return launch_pdl(grad_norm_kernel, dim3(1), dim3(OP_THREADS), 0, st, 1, used, partial, prescale, max_norm, out) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}
template <int CAP>
static int launch_grad_norm_with(const qlora_adamw_desc& d, float prescale, float max_norm, float* out, void* workspace, cudaStream_t st) {
    if (d.grad_type == QLORA_FP32) return launch_grad_norm_as<float, CAP>(d, prescale, max_norm, out, workspace, st);
    if (d.grad_type == QLORA_BF16) return launch_grad_norm_as<__nv_bfloat16, CAP>(d, prescale, max_norm, out, workspace, st);
    return launch_grad_norm_as<__half, CAP>(d, prescale, max_norm, out, workspace, st);
}

int launch_grad_norm(const qlora_adamw_desc& d, float prescale, float max_norm, float* out, void* workspace, cudaStream_t st) {
    if (d.n_tensors <= OP_SMALL_TABLE) return launch_grad_norm_with<OP_SMALL_TABLE>(d, prescale, max_norm, out, workspace, st);
    if (d.n_tensors <= OP_MIDDLE_TABLE) return launch_grad_norm_with<OP_MIDDLE_TABLE>(d, prescale, max_norm, out, workspace, st);
    return launch_grad_norm_with<OP_TABLE>(d, prescale, max_norm, out, workspace, st);
}

template <typename P, typename G, int CAP>
static cudaError_t launch_adamw_as(bool eight, uint32_t chunks, const OptTable<CAP>& tab, const AdamScalars& sc, cudaStream_t st) {
    if (eight) return launch_pdl(adamw_kernel<P, G, true, CAP>, dim3(chunks), dim3(OP_THREADS), 0, st, 1, tab, sc);
    return launch_pdl(adamw_kernel<P, G, false, CAP>, dim3(chunks), dim3(OP_THREADS), 0, st, 1, tab, sc);
}
template <typename P, int CAP>
static cudaError_t launch_adamw_param(int grad_type, bool eight, uint32_t chunks, const OptTable<CAP>& tab, const AdamScalars& sc, cudaStream_t st) {
    if (grad_type == QLORA_FP32) return launch_adamw_as<P, float>(eight, chunks, tab, sc, st);
    if (grad_type == QLORA_BF16) return launch_adamw_as<P, __nv_bfloat16>(eight, chunks, tab, sc, st);
    return launch_adamw_as<P, __half>(eight, chunks, tab, sc, st);
}
template <int CAP>
static int launch_adamw_with(const qlora_adamw_desc& d, const AdamScalars& sc, cudaStream_t st) {
    static thread_local OptTable<CAP> tab;
    int at = 0;
    for (;;) {
        const uint32_t chunks = fill_table(d, &at, tab);
        if (chunks == 0) return QLORA_OK;
        const bool eight = d.state_type == QLORA_E4M3;
        const cudaError_t err = d.param_type == QLORA_BF16 ? launch_adamw_param<__nv_bfloat16>(d.grad_type, eight, chunks, tab, sc, st)
                                : d.param_type == QLORA_FP16 ? launch_adamw_param<__half>(d.grad_type, eight, chunks, tab, sc, st)
                                                             : launch_adamw_param<float>(d.grad_type, eight, chunks, tab, sc, st);
        if (err != cudaSuccess) return QLORA_ERR_CUDA;
    }
}

int launch_adamw(const qlora_adamw_desc& d, double lr, int step, const float* lr_dev, const int32_t* step_dev, const float* norm, cudaStream_t st) {
    AdamScalars sc;
    sc.beta1 = (float)d.beta1; sc.one_minus_beta1 = (float)(1.0 - d.beta1);
    sc.beta2 = (float)d.beta2; sc.one_minus_beta2 = (float)(1.0 - d.beta2);
    sc.eps = (float)d.eps; sc.weight_decay = (float)d.weight_decay;
    sc.log_beta1 = (float)log(d.beta1); sc.log_beta2 = (float)log(d.beta2);
    sc.lr = (float)lr;
    sc.inv_corr1 = (float)(-1.0 / expm1(step * log(d.beta1))); sc.root_inv_corr2 = (float)(1.0 / sqrt(-expm1(step * log(d.beta2))));
    sc.step = step; sc.lr_dev = lr_dev; sc.step_dev = step_dev; sc.norm = norm;
    if (d.n_tensors <= OP_SMALL_TABLE) return launch_adamw_with<OP_SMALL_TABLE>(d, sc, st);
    if (d.n_tensors <= OP_MIDDLE_TABLE) return launch_adamw_with<OP_MIDDLE_TABLE>(d, sc, st);
    return launch_adamw_with<OP_TABLE>(d, sc, st);
}

}  // namespace qlora
