// Adapters of many requests beside one frozen projection.  Token t has an adapter a(t) in [0, L), or none:
//   down   P[t, :]   = In[t, :] L1_a                       (H = X A_a^T forward, G = dY B_a backward; zeros without an adapter)
//   up     Out[t, :] = Base[t, :] + s_a P[t, :] L2_a       (Y forward, dX backward)
//   grads  dA_a = s_a sum_{t in a} G[t]^T X[t],  dB_a = s_a sum_{t in a} dY[t]^T H[t]
// All of it is bound by memory: a rank is 8 to 64, so an element of In, Base or Out meets that many multiplications and no more.
//
// The adapters of a tile of tokens are found in the kernel, from the numbers of its tokens: entry e of a tile is one adapter and the bit
// mask of its tokens.  Nothing is planned ahead, so a call can be captured and replayed for another batch.  Every entry has sums of its
// own, from which only its own rows are taken: what an adapter holds (infinities, NaN) reaches its own tokens alone.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "device_state.h"
#include "launch.h"
#include "lora_down.cuh"
#include "tcgen05.cuh"

namespace qlora {
namespace {

typedef __nv_bfloat16 bf16;


__device__ __forceinline__ uint4 ldg16(const bf16* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// The entries of up to 32 tokens (lane i holds token i's adapter, -1 for none): lane i is the first token of an entry where it returns a
// mask, which names all tokens of that entry.
__device__ __forceinline__ uint32_t entry_of_lane(int adapter) {
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, adapter);
    const int lane = threadIdx.x & 31;
    return adapter >= 0 && (same & ((1u << lane) - 1u)) == 0 ? same : 0u;
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Two fp32 values as the sum of two bf16 each: products with both keep 16 bits of the value instead of 8.  The low part of what is not
// finite, or becomes so, is zero.
struct Split { uint32_t hi, lo; };
__device__ __forceinline__ Split split_bf16(float a, float b) {
    Split s;
    s.hi = bf16x2(a, b);
    const float la = a - bf16_lo(s.hi), lb = b - bf16_hi(s.hi);
    s.lo = bf16x2(fabsf(la) < INFINITY ? la : 0.f, fabsf(lb) < INFINITY ? lb : 0.f);
    return s;
}
// Zero in the place of infinities and NaN: what meets the low parts.  (Those have had their say in the product with the high part.)
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
    if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
    return w;
}

// ---------------------------------------------------------------------------------------------------------------- down
constexpr int DN_ROWS = 16, DN_SHARE = 4;

// One block per 16 tokens and DN_SHARE-th of their entries.  The warps stride over the contraction; fragments as in lora_down.cuh.
template <int NT> constexpr int DN_WARPS = NT <= 4 ? 16 : 8;             // (what 48 KB of shared memory hold of their sums)

template <bool L_IS_A, int NT>
__global__ void __launch_bounds__(32 * DN_WARPS<NT>)
adapters_down_kernel(int M, int T, int r, int n_adapters, const bf16* __restrict__ In, const int32_t* __restrict__ adapter_of,
                     const bf16* __restrict__ L, float* __restrict__ P) {
    constexpr int UNROLL = NT <= 2 ? 4 : NT <= 4 ? 2 : 1, WARPS = DN_WARPS<NT>;
    __shared__ float red[WARPS * NT * 128];
    __shared__ uint32_t entry_mask[DN_ROWS];
    __shared__ int entry_adapter[DN_ROWS], n_entries_s;
    __shared__ uint32_t bare_s;
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int m0 = blockIdx.x * DN_ROWS;
    if (warp == 0) {
        const bool in = lane < DN_ROWS && m0 + lane < M;
        int a = in ? adapter_of[m0 + lane] : -1;
        if (a < 0 || a >= n_adapters) a = -1;
        const uint32_t mask = entry_of_lane(a);
        const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mask != 0), bare = __ballot_sync(0xFFFFFFFFu, in && a < 0);
        if (mask != 0) {
            const int e = __popc(firsts & ((1u << lane) - 1u));
            entry_mask[e] = mask;
            entry_adapter[e] = a;
        }
        if (lane == 0) { n_entries_s = __popc(firsts); bare_s = bare; }
    }
    __syncthreads();
    if (blockIdx.y == 0) {
        for (int i = threadIdx.x; i < DN_ROWS * r; i += 32 * WARPS)
            if ((bare_s >> (i / r)) & 1u) P[(size_t)m0 * r + i] = 0.f;
    }
    const int n_entries = n_entries_s;
    const uint4 zero4 = make_uint4(0, 0, 0, 0);
    for (int e = blockIdx.y; e < n_entries; e += DN_SHARE) {
        const uint32_t mask = entry_mask[e];
        const bf16* La = L + (size_t)entry_adapter[e] * r * T;
        const bool on0 = (mask >> g) & 1u, on1 = (mask >> (g + 8)) & 1u;
        const bf16 *x0 = In + (size_t)(m0 + g) * T, *x1 = x0 + (size_t)8 * T;
        float acc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
#pragma unroll 1
        for (int kk = warp * 32; kk < T; kk += WARPS * 32 * UNROLL) {
            uint4 xlo[UNROLL], xhi[UNROLL], l[UNROLL][NT];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int k0 = kk + u * WARPS * 32, k = k0 + q * 8;
                xlo[u] = on0 && k < T ? ldg16(x0 + k) : zero4;
                xhi[u] = on1 && k < T ? ldg16(x1 + k) : zero4;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint4 lv = zero4;
                    if (L_IS_A) {
                        const int j = nt * 8 + g;
                        if (k < T && j < r) lv = ldg16(La + (size_t)j * T + k);
                    } else if (nt * 8 < r) {
                        const int n = k0 + 8 * (g >> 1) + (g & 1);
                        const uint32_t* src = reinterpret_cast<const uint32_t*>(La + (size_t)n * r + nt * 8 + 2 * q);
                        if (n < T) lv = make_uint4(__ldg(src), __ldg(src + r), __ldg(src + 2 * r), __ldg(src + 3 * r));
                    }
                    l[u][nt] = lv;
                }
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                if (kk + u * WARPS * 32 >= T) break;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint4 lv = l[u][nt];
                    if (!L_IS_A) lv = make_uint4(movmatrix_trans(lv.x), movmatrix_trans(lv.y), movmatrix_trans(lv.z), movmatrix_trans(lv.w));
                    mma_bf16_16816(acc[nt], xlo[u].x, xhi[u].x, xlo[u].y, xhi[u].y, lv.x, lv.y);
                    mma_bf16_16816(acc[nt], xlo[u].z, xhi[u].z, xlo[u].w, xhi[u].w, lv.z, lv.w);
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) red[((warp * NT + nt) * 4 + c) * 32 + lane] = acc[nt][c];
        __syncthreads();
        for (int idx = threadIdx.x; idx < NT * 128; idx += 32 * WARPS) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += red[w * NT * 128 + idx];
            const int nt = idx >> 7, c = (idx >> 5) & 3, ln = idx & 31;
            const int row = (ln >> 2) + ((c & 2) ? 8 : 0), col = nt * 8 + (ln & 3) * 2 + (c & 1);
            if (((mask >> row) & 1u) && col < r) P[(size_t)(m0 + row) * r + col] = v;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------------------ up
constexpr int UP_ROWS = 16, UP_WARPS = 8, UP_BLOCKS = 2;               // a warp: 16 tokens x 2 blocks of 32 columns

// The adapter's part for 32 columns (c0 ..) and ranks 16 ks .. 16 ks + 15 as four column tiles of an MMA.  Column c of tile t is
// c0 + 8 (c / 2) + 2 t + c % 2, so a thread's sums are eight neighbouring columns.  FROM_B: L2 = B [C, r]; else A [r, C].  The ranks are in the order
// (4 q, 4 q + 1; 4 q + 2, 4 q + 3) for B, which is read along them, and (2 q, 2 q + 1; 8 + 2 q, 9 + 2 q) for A.
template <bool FROM_B>
__device__ __forceinline__ void up_fragments(const bf16* __restrict__ L2, int C, int r, int c0, int ks, int g, int q, uint32_t (&b)[4][2]) {
    if constexpr (FROM_B) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int n = c0 + 8 * (g >> 1) + 2 * t + (g & 1), j = 16 * ks + 4 * q;
            uint2 v = make_uint2(0, 0);
            if (n < C && j < r) v = __ldg(reinterpret_cast<const uint2*>(L2 + (size_t)n * r + j));
            b[t][0] = v.x;
            b[t][1] = v.y;
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = 16 * ks + 8 * h + g, n = c0 + 8 * q;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (n < C && j < r) v = ldg16(L2 + (size_t)j * C + n);
            b[0][h] = movmatrix_trans(v.x);
            b[1][h] = movmatrix_trans(v.y);
            b[2][h] = movmatrix_trans(v.z);
            b[3][h] = movmatrix_trans(v.w);
        }
    }
}

template <bool FROM_B>
__global__ void __launch_bounds__(32 * UP_WARPS)
adapters_up_kernel(int M, int C, int r, int n_adapters, const float* __restrict__ P, const int32_t* __restrict__ adapter_of,
                   const bf16* __restrict__ L, const float* __restrict__ scales, const bf16* Base, bf16* Out) {
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int m0 = blockIdx.x * UP_ROWS, c_warp = (blockIdx.y * UP_WARPS + warp) * 32 * UP_BLOCKS;
    if (c_warp >= C) return;
    int a = lane < UP_ROWS && m0 + lane < M ? adapter_of[m0 + lane] : -1;
    if (a < 0 || a >= n_adapters) a = -1;
    const uint32_t mask_here = entry_of_lane(a);
    uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mask_here != 0);
    const int row0 = m0 + g, row1 = row0 + 8;
    uint4 base[UP_BLOCKS][2];
#pragma unroll
    for (int i = 0; i < UP_BLOCKS; ++i) {
        const int c = c_warp + 32 * i + 8 * q;
        const uint4 zero4 = make_uint4(0, 0, 0, 0);
        base[i][0] = row0 < M && c < C ? *reinterpret_cast<const uint4*>(Base + (size_t)row0 * C + c) : zero4;
        base[i][1] = row1 < M && c < C ? *reinterpret_cast<const uint4*>(Base + (size_t)row1 * C + c) : zero4;
    }
    float sum[UP_BLOCKS][4][4] = {};
    while (firsts != 0) {
        const int first = __ffs(firsts) - 1;
        firsts &= firsts - 1;
        const uint32_t mask = __shfl_sync(0xFFFFFFFFu, mask_here, first);
        const int adapter = __shfl_sync(0xFFFFFFFFu, a, first);
        const bool on0 = (mask >> g) & 1u, on1 = (mask >> (g + 8)) & 1u;
        const float s = scales[adapter];
        const bf16* L2 = L + (size_t)adapter * r * C;
        float part[UP_BLOCKS][4][4] = {};
        for (int ks = 0; 16 * ks < r; ++ks) {
            // the tokens' part: s P of ranks in the adapter's order, as two bf16 each
            float2 p[2][2];                                            // [row][half]
            const int j0 = FROM_B ? 16 * ks + 4 * q : 16 * ks + 2 * q, j1 = FROM_B ? j0 + 2 : j0 + 8;
            const float2 none = make_float2(0.f, 0.f);
            p[0][0] = on0 && j0 < r ? __ldcg(reinterpret_cast<const float2*>(P + (size_t)row0 * r + j0)) : none;
            p[1][0] = on1 && j0 < r ? __ldcg(reinterpret_cast<const float2*>(P + (size_t)row1 * r + j0)) : none;
            p[0][1] = on0 && j1 < r ? __ldcg(reinterpret_cast<const float2*>(P + (size_t)row0 * r + j1)) : none;
            p[1][1] = on1 && j1 < r ? __ldcg(reinterpret_cast<const float2*>(P + (size_t)row1 * r + j1)) : none;
            Split x[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[i][h] = split_bf16(s * p[i][h].x, s * p[i][h].y);
#pragma unroll
            for (int i = 0; i < UP_BLOCKS; ++i) {
                uint32_t b[4][2];
                up_fragments<FROM_B>(L2, C, r, c_warp + 32 * i, ks, g, q, b);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    mma_bf16_16816(part[i][t], x[0][0].hi, x[1][0].hi, x[0][1].hi, x[1][1].hi, b[t][0], b[t][1]);
                    mma_bf16_16816(part[i][t], x[0][0].lo, x[1][0].lo, x[0][1].lo, x[1][1].lo, finite_pair(b[t][0]), finite_pair(b[t][1]));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < UP_BLOCKS; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (on0) { sum[i][t][0] = part[i][t][0]; sum[i][t][1] = part[i][t][1]; }
                if (on1) { sum[i][t][2] = part[i][t][2]; sum[i][t][3] = part[i][t][3]; }
            }
    }
    const bool any0 = __shfl_sync(0xFFFFFFFFu, a, g) >= 0, any1 = __shfl_sync(0xFFFFFFFFu, a, g + 8) >= 0;
#pragma unroll
    for (int i = 0; i < UP_BLOCKS; ++i) {
        const int c = c_warp + 32 * i + 8 * q;
        if (c >= C) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = h ? row1 : row0;
            if (row >= M) continue;
            uint4 v = base[i][h];
            if (h ? any1 : any0) {                                     // (a token without an adapter keeps its bits, whatever they are)
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int t = 0; t < 4; ++t) w[t] = bf16x2(bf16_lo(w[t]) + sum[i][t][2 * h], bf16_hi(w[t]) + sum[i][t][2 * h + 1]);
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4*>(Out + (size_t)row * C + c) = v;
        }
    }
}

// ----------------------------------------------------------------------------------------------------------- few tokens
constexpr int FEW_ROWS = 4, FEW_CTAS = 8, FEW_WARPS = 8;

// Both products of FEW_ROWS tokens in one launch, by a cluster.  Its CTAs share the contraction out; each stores its sums into the shared memory
// of all, and one cluster barrier later they share the columns out.  The adapters' second matrices are asked into L2 before the first product
// begins.  The second product is fp32 throughout: a few tokens leave the CUDA cores enough time.
template <bool FORWARD, int NT>
__global__ void __cluster_dims__(FEW_CTAS, 1, 1) __launch_bounds__(32 * FEW_WARPS)
adapters_few_kernel(int M, int T, int C, int r, int n_adapters, const bf16* __restrict__ In, const int32_t* __restrict__ adapter_of,
                    const bf16* __restrict__ L1, const bf16* __restrict__ L2, const float* __restrict__ scales, const bf16* Base, bf16* Out,
                    float* __restrict__ P_out) {
    constexpr int UNROLL = NT <= 2 ? 4 : NT <= 4 ? 2 : 1, THREADS = 32 * FEW_WARPS;
    __shared__ float red[FEW_WARPS][FEW_ROWS][NT * 8];
    __shared__ __align__(16) float parts[FEW_CTAS][FEW_ROWS][NT * 8];  // [CTA that summed]
    __shared__ __align__(16) float low[FEW_ROWS][NT * 8];              // s P
    __shared__ uint32_t entry_mask[FEW_ROWS];
    __shared__ int entry_adapter[FEW_ROWS], entry_of[FEW_ROWS], n_entries_s;
    pdl_launch_dependents();
    cluster_arrive();                                                  // (a CTA's shared memory is written to once it has begun)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int cta = (int)cluster_ctarank(), m0 = (int)(blockIdx.x / FEW_CTAS) * FEW_ROWS, rows = min(FEW_ROWS, M - m0);
    pdl_wait();
    if (warp == 0) {
        int a = lane < rows ? adapter_of[m0 + lane] : -1;
        if (a < 0 || a >= n_adapters) a = -1;
        const uint32_t mask = entry_of_lane(a), firsts = __ballot_sync(0xFFFFFFFFu, mask != 0);
        const int first = __ffs(__match_any_sync(0xFFFFFFFFu, a)) - 1, e = __popc(firsts & ((1u << (a >= 0 ? first : 0)) - 1u));
        if (lane < FEW_ROWS) entry_of[lane] = a >= 0 ? e : -1;
        if (mask != 0) { entry_mask[e] = mask; entry_adapter[e] = a; }
        if (lane == 0) n_entries_s = __popc(firsts);
    }
    __syncthreads();
    const int n_entries = n_entries_s, pairs = C / 2;
    const int p_lo = (int)((long long)pairs * cta / FEW_CTAS), p_hi = (int)((long long)pairs * (cta + 1) / FEW_CTAS);
    for (int e = 0; e < n_entries; ++e) {
        const bf16* La = L2 + (size_t)entry_adapter[e] * r * C;
        if constexpr (FORWARD) {                                       // B: the columns' rows lie together
            for (int i = p_lo * 2 * r + 64 * threadIdx.x; i < p_hi * 2 * r; i += 64 * THREADS) asm volatile("prefetch.global.L2 [%0];" ::"l"(La + i));
        } else {
            const int lines = (p_hi - p_lo + 31) / 32;
            for (int i = threadIdx.x; i < lines * r; i += THREADS)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(La + (size_t)(i / lines) * C + 2 * p_lo + 64 * (i % lines)));
        }
    }
    // ---- the first product: warps share the entries and their parts of the contraction
    const int per_entry = n_entries <= 1 ? 8 : n_entries == 2 ? 4 : 2, my_entry = warp / per_entry, sub = warp % per_entry;
    if (my_entry < n_entries) {
        const int steps = (T + 31) / 32, s_lo = steps * cta / FEW_CTAS, s_hi = steps * (cta + 1) / FEW_CTAS;
        const bf16* La = L1 + (size_t)entry_adapter[my_entry] * r * T;
        const bool on = g < FEW_ROWS && ((entry_mask[my_entry] >> g) & 1u);
        const bf16* x0 = In + (size_t)(m0 + g) * T;
        const uint4 zero4 = make_uint4(0, 0, 0, 0);
        float acc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
#pragma unroll 1
        for (int step = s_lo + sub; step < s_hi; step += per_entry * UNROLL) {
            uint4 x[UNROLL], l[UNROLL][NT];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int at = step + u * per_entry, k0 = 32 * at, k = k0 + q * 8;
                const bool in = at < s_hi;
                x[u] = in && on && k < T ? ldg16(x0 + k) : zero4;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint4 lv = zero4;
                    if (FORWARD) {
                        const int j = nt * 8 + g;
                        if (in && k < T && j < r) lv = ldg16(La + (size_t)j * T + k);
                    } else if (nt * 8 < r) {
                        const int n = k0 + 8 * (g >> 1) + (g & 1);
                        const uint32_t* src = reinterpret_cast<const uint32_t*>(La + (size_t)n * r + nt * 8 + 2 * q);
                        if (in && n < T) lv = make_uint4(__ldg(src), __ldg(src + r), __ldg(src + 2 * r), __ldg(src + 3 * r));
                    }
                    l[u][nt] = lv;
                }
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint4 lv = l[u][nt];
                    if (!FORWARD) lv = make_uint4(movmatrix_trans(lv.x), movmatrix_trans(lv.y), movmatrix_trans(lv.z), movmatrix_trans(lv.w));
                    mma_bf16_16816(acc[nt], x[u].x, 0u, x[u].y, 0u, lv.x, lv.y);
                    mma_bf16_16816(acc[nt], x[u].z, 0u, x[u].w, 0u, lv.z, lv.w);
                }
        }
        if (g < FEW_ROWS)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                red[warp][g][nt * 8 + 2 * q] = acc[nt][0];
                red[warp][g][nt * 8 + 2 * q + 1] = acc[nt][1];
            }
    }
    __syncthreads();
    cluster_wait();                                                    // every CTA of the cluster has begun
    if (threadIdx.x < FEW_ROWS * NT * 8) {
        const int row = threadIdx.x / (NT * 8), j = threadIdx.x % (NT * 8), e = row < rows ? entry_of[row] : -1;
        float v = 0.f;
        if (e >= 0)
            for (int w = 0; w < per_entry; ++w) v += red[e * per_entry + w][row][j];
        const uint32_t here = (uint32_t)__cvta_generic_to_shared(&parts[cta][row][j]);
#pragma unroll
        for (int i = 0; i < FEW_CTAS; ++i) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(here, i)), "f"(v) : "memory");
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (threadIdx.x < FEW_ROWS * NT * 8) {
        const int row = threadIdx.x / (NT * 8), j = threadIdx.x % (NT * 8), e = row < rows ? entry_of[row] : -1;
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < FEW_CTAS; ++i) v += parts[i][row][j];
        if (P_out != nullptr && cta == 0 && row < rows && j < r) P_out[(size_t)(m0 + row) * r + j] = v;
        low[row][j] = e >= 0 ? scales[entry_adapter[e]] * v : 0.f;
    }
    __syncthreads();
    // ---- the second product: a thread has two neighbouring columns of one entry
    const int n_pairs = p_hi - p_lo;
    for (int unit = threadIdx.x; unit < n_entries * n_pairs; unit += THREADS) {
        const int e = unit / n_pairs, c = 2 * (p_lo + unit - e * n_pairs);
        const bf16* La = L2 + (size_t)entry_adapter[e] * r * C;
        const uint32_t mask = entry_mask[e];
        float sum[FEW_ROWS][2] = {};
        uint32_t base[FEW_ROWS];
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i)
            base[i] = (mask >> i) & 1u ? *reinterpret_cast<const uint32_t*>(Base + (size_t)(m0 + i) * C + c) : 0u;
#pragma unroll
        for (int j = 0; j < NT * 8; j += 8) {
            if (j >= r) break;
            float w[8][2];                                             // eight ranks of both columns
            if constexpr (FORWARD) {
                const uint4 a = ldg16(La + (size_t)c * r + j), b = ldg16(La + (size_t)(c + 1) * r + j);
                const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i][0] = i & 1 ? bf16_hi(wa[i / 2]) : bf16_lo(wa[i / 2]);
                    w[i][1] = i & 1 ? bf16_hi(wb[i / 2]) : bf16_lo(wb[i / 2]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t a = __ldg(reinterpret_cast<const uint32_t*>(La + (size_t)(j + i) * C + c));
                    w[i][0] = bf16_lo(a);
                    w[i][1] = bf16_hi(a);
                }
            }
#pragma unroll
            for (int i = 0; i < FEW_ROWS; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float p = low[i][j + k];
                    sum[i][0] = fmaf(p, w[k][0], sum[i][0]);
                    sum[i][1] = fmaf(p, w[k][1], sum[i][1]);
                }
        }
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i)
            if ((mask >> i) & 1u)
                *reinterpret_cast<uint32_t*>(Out + (size_t)(m0 + i) * C + c) = bf16x2(bf16_lo(base[i]) + sum[i][0], bf16_hi(base[i]) + sum[i][1]);
    }
    if (Out != Base)                                                   // tokens without an adapter
        for (int i = 0; i < rows; ++i)
            if (entry_of[i] < 0)
                for (int p = p_lo + threadIdx.x; p < p_hi; p += THREADS)
                    *reinterpret_cast<uint32_t*>(Out + (size_t)(m0 + i) * C + 2 * p) = *reinterpret_cast<const uint32_t*>(Base + (size_t)(m0 + i) * C + 2 * p);
}

// --------------------------------------------------------------------------------------------------------------- grads
constexpr int GR_WARPS = 8, GR_WINDOW = 2048;

// One block per adapter and slice of 32 NB columns of X (then of dY): the block finds its adapter's tokens, window by window, in the order
// of their places; its warps take sixteen of them at a time, and their sums are added in the order of the warps.  MT tiles of 16 ranks.
template <int MT, int NB>
__global__ void __launch_bounds__(32 * GR_WARPS)
adapters_grad_kernel(int M, int K, int N, int r, int n_adapters, const bf16* __restrict__ X, const bf16* __restrict__ dY,
                     const int32_t* __restrict__ adapter_of, const float* __restrict__ scales, const float* __restrict__ H, const float* __restrict__ G,
                     float* __restrict__ dA, float* __restrict__ dB, int accumulate) {
    extern __shared__ float red[];                                     // [warps][MT * 16][32 NB]
    __shared__ int list[GR_WINDOW];
    __shared__ int counts[GR_WARPS];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int adapter = blockIdx.y, slices_x = (K + 32 * NB - 1) / (32 * NB);
    const bool of_x = (int)blockIdx.x < slices_x;
    const int C = of_x ? K : N, c0 = (of_x ? blockIdx.x : blockIdx.x - slices_x) * 32 * NB;
    const bf16* V = of_x ? X : dY;
    const float* P = of_x ? G : H;
    float acc[MT][NB][4][4] = {};
    bool any = false;
    for (int w0 = 0; w0 < M; w0 += GR_WINDOW) {
        // this warp's share of the window: GR_WINDOW / GR_WARPS places in a row
        constexpr int SHARE = GR_WINDOW / GR_WARPS;
        const int from = w0 + warp * SHARE;
        uint32_t found[SHARE / 32];
        int n = 0;
#pragma unroll
        for (int i = 0; i < SHARE / 32; ++i) {
            const int t = from + 32 * i + lane;
            found[i] = __ballot_sync(0xFFFFFFFFu, t < M && __ldg(adapter_of + t) == adapter);
            n += __popc(found[i]);
        }
        if (lane == 0) counts[warp] = n;
        __syncthreads();
        int at = 0, total = 0;
#pragma unroll
        for (int w = 0; w < GR_WARPS; ++w) {
            if (w == warp) at = total;
            total += counts[w];
        }
#pragma unroll
        for (int i = 0; i < SHARE / 32; ++i) {
            if ((found[i] >> lane) & 1u) list[at + __popc(found[i] & ((1u << lane) - 1u))] = from + 32 * i + lane;
            at += __popc(found[i]);
        }
        __syncthreads();
        any |= total > 0;
        for (int i0 = warp * 16; i0 < total; i0 += GR_WARPS * 16) {
            // tokens i0 + g and i0 + 8 + g in rows of 32 columns; after the transposition a thread has tokens 2 q, 2 q + 1 (+ 8) of one column
            uint32_t b[NB][4][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = i0 + 8 * h + g;
                const bf16* row = i < total ? V + (size_t)list[i] * C : nullptr;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int c = c0 + 32 * nb + 8 * q;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (row != nullptr && c < C) v = ldg16(row + c);
                    b[nb][0][h] = v.x; b[nb][1][h] = v.y; b[nb][2][h] = v.z; b[nb][3][h] = v.w;
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    b[nb][t][0] = movmatrix_trans(b[nb][t][0]);
                    b[nb][t][1] = movmatrix_trans(b[nb][t][1]);
                }
            const float* pt[4];                                        // rows of P of tokens 2 q, 2 q + 1, 8 + 2 q, 9 + 2 q
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + 2 * q + (k & 1) + 8 * (k >> 1);
                pt[k] = i < total ? P + (size_t)list[i] * r : nullptr;
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                Split p[2][2];                                         // [rank half][token half]
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int j = 16 * mt + 8 * i + g;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        p[i][h] = split_bf16(pt[2 * h] && j < r ? __ldg(pt[2 * h] + j) : 0.f, pt[2 * h + 1] && j < r ? __ldg(pt[2 * h + 1] + j) : 0.f);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        mma_bf16_16816(acc[mt][nb][t], p[0][0].hi, p[1][0].hi, p[0][1].hi, p[1][1].hi, b[nb][t][0], b[nb][t][1]);
                        mma_bf16_16816(acc[mt][nb][t], p[0][0].lo, p[1][0].lo, p[0][1].lo, p[1][1].lo, finite_pair(b[nb][t][0]), finite_pair(b[nb][t][1]));
                    }
            }
        }
        __syncthreads();                                               // the list is written again
    }
    if (!any && accumulate) return;                                    // (the same for the whole block)
    // acc[mt][nb][t][c]: rank 16 mt + g (+ 8 where c >= 2), column 32 nb + 8 q + 2 t + c % 2
    constexpr int COLS = 32 * NB;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(red + ((size_t)warp * MT * 16 + 16 * mt + 8 * h + g) * COLS + 32 * nb + 8 * q + 2 * t) =
                        make_float2(acc[mt][nb][t][2 * h], acc[mt][nb][t][2 * h + 1]);
    __syncthreads();
    const float s = scales[adapter];
    for (int idx = threadIdx.x; idx < r * COLS; idx += 32 * GR_WARPS) {
        // in the order of the output: A's gradient along the columns, B's along the ranks
        const int j = of_x ? idx / COLS : idx % r, c = of_x ? idx % COLS : idx / r;
        if (c0 + c >= C) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < GR_WARPS; ++w) v += red[((size_t)w * MT * 16 + j) * COLS + c];
        float* dst = of_x ? dA + ((size_t)adapter * r + j) * K + c0 + c : dB + ((size_t)adapter * N + c0 + c) * r + j;
        v = any ? s * v : 0.f;
        *dst = accumulate ? *dst + v : v;
    }
}

template <bool L_IS_A, int NT>
int down_impl(int M, int T, int r, int n_adapters, const void* In, const int32_t* adapter_of, const void* L, float* P, cudaStream_t st) {
    return launch_pdl(adapters_down_kernel<L_IS_A, NT>, dim3((M + DN_ROWS - 1) / DN_ROWS, DN_SHARE), dim3(32 * DN_WARPS<NT>), 0, st, 1, M, T, r, n_adapters,
                      (const bf16*)In, adapter_of, (const bf16*)L, P) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

template <bool FORWARD, int NT>
int few_impl(int M, int T, int C, int r, int L, const void* In, const int32_t* adapter_of, const void* L1, const void* L2, const float* scales,
             const void* Base, void* Out, float* P_out, cudaStream_t st) {
    return launch_pdl(adapters_few_kernel<FORWARD, NT>, dim3((M + FEW_ROWS - 1) / FEW_ROWS * FEW_CTAS), dim3(32 * FEW_WARPS), 0, st, 1, M, T, C, r, L,
                      (const bf16*)In, adapter_of, (const bf16*)L1, (const bf16*)L2, scales, (const bf16*)Base, (bf16*)Out, P_out) == cudaSuccess
               ? QLORA_OK : QLORA_ERR_CUDA;   // (the cluster's width is an attribute of the kernel)
}

template <int MT, int NB>
int grad_impl(int M, int K, int N, int r, int L, const void* X, const void* dY, const int32_t* adapter_of, const float* scales, const float* H,
              const float* G, float* dA, float* dB, int accumulate, cudaStream_t st) {
    constexpr size_t smem = sizeof(float) * GR_WARPS * MT * 16 * 32 * NB;
    static SmemLimit limit;
    auto kern = adapters_grad_kernel<MT, NB>;
    if (!limit.raise(kern, smem)) return QLORA_ERR_CUDA;
    const int slices = (K + 32 * NB - 1) / (32 * NB) + (N + 32 * NB - 1) / (32 * NB);
    return launch_pdl(kern, dim3(slices, L), dim3(32 * GR_WARPS), smem, st, 1, M, K, N, r, L, (const bf16*)X, (const bf16*)dY, adapter_of, scales, H, G,
                      dA, dB, accumulate) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

}  // namespace

int launch_adapters_down(int M, int T, int r, int n_adapters, bool l_is_A, const void* In, const int32_t* adapter_of, const void* L, float* P, cudaStream_t st) {
#define QLORA_DOWN(NT) return l_is_A ? down_impl<true, NT>(M, T, r, n_adapters, In, adapter_of, L, P, st) : down_impl<false, NT>(M, T, r, n_adapters, In, adapter_of, L, P, st)
    if (r <= 8) QLORA_DOWN(1);
    if (r <= 16) QLORA_DOWN(2);
    if (r <= 32) QLORA_DOWN(4);
    QLORA_DOWN(8);
#undef QLORA_DOWN
}

int launch_adapters_up(int M, int C, int r, int n_adapters, bool from_B, const float* P, const int32_t* adapter_of, const void* L, const float* scales,
                       const void* Base, void* Out, cudaStream_t st) {
    const dim3 grid((M + UP_ROWS - 1) / UP_ROWS, (C + 32 * UP_BLOCKS * UP_WARPS - 1) / (32 * UP_BLOCKS * UP_WARPS));
    return launch_pdl(from_B ? adapters_up_kernel<true> : adapters_up_kernel<false>, grid, dim3(32 * UP_WARPS), 0, st, 1, M, C, r, n_adapters, P, adapter_of,
                      (const bf16*)L, scales, (const bf16*)Base, (bf16*)Out) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

bool adapters_few(int M) { return M <= 256; }

int launch_adapters_few(int M, int T, int C, int r, int n_adapters, bool forward, const void* In, const int32_t* adapter_of, const void* L1, const void* L2,
                        const float* scales, const void* Base, void* Out, float* P_out, cudaStream_t st) {
#define QLORA_FEW(NT)                                                                                                               \
    return forward ? few_impl<true, NT>(M, T, C, r, n_adapters, In, adapter_of, L1, L2, scales, Base, Out, P_out, st)              \
                   : few_impl<false, NT>(M, T, C, r, n_adapters, In, adapter_of, L1, L2, scales, Base, Out, P_out, st)
    if (r <= 8) QLORA_FEW(1);
    if (r <= 16) QLORA_FEW(2);
    if (r <= 32) QLORA_FEW(4);
    QLORA_FEW(8);
#undef QLORA_FEW
}

int launch_adapters_grads(int M, int K, int N, int r, int n_adapters, const void* X, const void* dY, const int32_t* adapter_of, const float* scales,
                          const float* H, const float* G, float* dA, float* dB, int accumulate, cudaStream_t st) {
#define QLORA_GRAD(MT, NB) return grad_impl<MT, NB>(M, K, N, r, n_adapters, X, dY, adapter_of, scales, H, G, dA, dB, accumulate, st)
    if (r <= 16) QLORA_GRAD(1, 2);
    if (r <= 32) QLORA_GRAD(2, 1);
    QLORA_GRAD(4, 1);
#undef QLORA_GRAD
}

}  // namespace qlora
