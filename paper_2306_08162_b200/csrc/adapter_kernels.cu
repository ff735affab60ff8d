// Adapters of many requests beside one frozen projection.  Token t has an adapter a(t) in [0, L), or none:
//   down   P[t, :]   = In[t, :] L1_a                       (H = X A_a^T forward, G = dY B_a backward; zeros without an adapter)
//   up     Out[t, :] = Base[t, :] + s_a P[t, :] L2_a       (Y forward, dX backward)
//   grads  dA_a = s_a sum_{t in a} G[t]^T X[t],  dB_a = s_a sum_{t in a} dY[t]^T H[t]
// All of it is bound by memory: a rank is 8 to 64, so an element of In, Base or Out meets that many multiplications and no more.
//
// Which adapters a tile of tokens has is found on the device, from the numbers of its tokens: entry e of a tile is one adapter and the bit
// mask of its tokens.  The host plans nothing, so a call can be captured and replayed for another batch.  Every entry has sums of its
// own, from which only its own rows are taken: what an adapter holds (infinities, NaN) reaches its own tokens alone.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// 16 bytes to shared memory, zeros where `in` is false; groups of such copies; 8 x 8 matrices out of it, as they lie or transposed.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    if constexpr (TRANS) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr));
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr));
}

// ----------------------------------------------------------------------------------------------------------- few tokens
// Both products of ROWS tokens by a cluster (or one block).  Its CTAs share the contraction out; each stores its sums into the shared memory of all, and one cluster
// barrier later they share the columns out.  The adapters' second matrices are asked into L2 before the first product begins.  The second product
// is fp32 throughout: a few tokens leave the CUDA cores enough time.
// Bound by latency: asking, products, the exchange, the second asking and the store, one after the other.  One token, rank 16, 4096 x 4096: 8.3 us a call (which is
// what the host takes to issue it); 64 tokens of 64 adapters, 4096 x 11008: 10.7 us for 30 MB, 2.8 TB/s.
constexpr int FEW_WARPS = 8, FEW_TOKENS = 256;

template <int NT, int ROWS, int CTAS>
struct FewShared {
    float parts[CTAS][ROWS][NT * 8];                               // [CTA that summed]
    float red[FEW_WARPS][ROWS][NT * 8];
    float low[ROWS][NT * 8];                                           // s P
    uint32_t entry_mask[ROWS];
    int entry_adapter[ROWS], entry_of[ROWS], n_entries;
};

// Tokens that are taken out of their tiles (see `adapters_groups_kernel`), up to 16 of one adapter in a group.
constexpr int GROUP = 16, NO_ADAPTER = 0xFFFF;
struct Groups {
    int* head;                               // [0] groups, [1] claimed
    int2* groups;                            // [M]: place in `tokens` << 5 | how many; adapter, or NO_ADAPTER
    int* tokens;                             // [M]
};

// A row of s P in parts: sixteen ranks at a time, in the order in which the second product's lanes take them, 16 bytes each (`up_low`).
constexpr __host__ __device__ int split_pairs(int r) { return (r + 15) / 16 * 8; }

struct Products {                            // the operands of both products
    int M, T, C, r, n_adapters;
    const bf16* In;                          // [M, T]
    const int32_t* adapter_of;
    const bf16 *L1, *L2;                     // forward: A, B; else B, A
    const float* scales;
    const bf16* Base;                        // [M, C]; no second product where Out is NULL
    bf16* Out;
    float* P;                                // [M, r] or NULL
    uint2* split;                            // [M, split_pairs(r)]: pairs of s P as two bf16 pairs, for the second product of many tokens; or NULL
    Groups groups;                           // of many tokens
};

// Called by all threads of all CTAs of the cluster, with the same m0, after the cluster's CTAs have begun.
template <bool FORWARD, int NT, int ROWS, int CTAS>
__device__ __forceinline__ void few_tokens(const Products& p, int m0, FewShared<NT, ROWS, CTAS>& sh) {
    constexpr int UNROLL = NT <= 2 ? 4 : NT <= 4 ? 2 : 1, THREADS = 32 * FEW_WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int cta = CTAS > 1 ? (int)cluster_ctarank() : 0, rows = min(ROWS, p.M - m0), r = p.r, T = p.T, C = p.C;
    if (warp == 0) {
        int a = lane < rows ? p.adapter_of[m0 + lane] : -1;
        if (a < 0 || a >= p.n_adapters) a = -1;
        const uint32_t mask = entry_of_lane(a), firsts = __ballot_sync(0xFFFFFFFFu, mask != 0);
        const int first = __ffs(__match_any_sync(0xFFFFFFFFu, a)) - 1, e = __popc(firsts & ((1u << (a >= 0 ? first : 0)) - 1u));
        if (lane < ROWS) sh.entry_of[lane] = a >= 0 ? e : -1;
        if (mask != 0) { sh.entry_mask[e] = mask; sh.entry_adapter[e] = a; }
        if (lane == 0) sh.n_entries = __popc(firsts);
    }
    __syncthreads();
    const int n_entries = sh.n_entries, pairs = C / 2;
    const int p_lo = (int)((long long)pairs * cta / CTAS), p_hi = (int)((long long)pairs * (cta + 1) / CTAS);
    for (int e = 0; e < n_entries; ++e) {
        const bf16* La = p.L2 + (size_t)sh.entry_adapter[e] * r * C;
        if constexpr (FORWARD) {                                       // B: the columns' rows lie together
            for (int i = p_lo * 2 * r + 64 * threadIdx.x; i < p_hi * 2 * r; i += 64 * THREADS) prefetch_l2(La + i);
        } else {
            const int lines = (p_hi - p_lo + 31) / 32;
            for (int i = threadIdx.x; i < lines * r; i += THREADS) prefetch_l2(La + (size_t)(i / lines) * C + 2 * p_lo + 64 * (i % lines));
        }
    }
    // ---- the first product: warps share the entries and their parts of the contraction.  (A row of the result depends on its own row of In alone, so
    // rows of other entries need no mask: they are not taken.)
    const int per_entry = n_entries <= 1 ? 8 : n_entries == 2 ? 4 : 2, my_entry = warp / per_entry, sub = warp % per_entry;
    if (my_entry < n_entries) {
        const int steps = (T + 31) / 32, s_lo = steps * cta / CTAS, s_hi = steps * (cta + 1) / CTAS;
        const bf16* La = p.L1 + (size_t)sh.entry_adapter[my_entry] * r * T;
        const bool on = g < rows;
        const bf16* x0 = p.In + (size_t)(m0 + g) * T;
        const uint4 zero4 = make_uint4(0, 0, 0, 0);
        float acc[NT][4] = {};
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
        if (g < ROWS)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<float2*>(&sh.red[warp][g][nt * 8 + 2 * q]) = make_float2(acc[nt][0], acc[nt][1]);
    }
    __syncthreads();
    constexpr int VALUES = ROWS * NT * 8;
    if (threadIdx.x < VALUES) {
        const int row = threadIdx.x / (NT * 8), j = threadIdx.x % (NT * 8), e = row < rows ? sh.entry_of[row] : -1;
        float v = 0.f;
        if (e >= 0)
            for (int w = 0; w < per_entry; ++w) v += sh.red[e * per_entry + w][row][j];
        if constexpr (CTAS > 1) {
            const uint32_t here = smem_u32(&sh.parts[cta][row][j]);
#pragma unroll
            for (int i = 0; i < CTAS; ++i) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(here, i)), "f"(v) : "memory");
        } else {
            sh.parts[0][row][j] = v;                                   // (read by the thread that wrote it)
        }
    }
    if constexpr (CTAS > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (threadIdx.x < VALUES) {
        const int row = threadIdx.x / (NT * 8), j = threadIdx.x % (NT * 8), e = row < rows ? sh.entry_of[row] : -1;
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < CTAS; ++i) v += sh.parts[i][row][j];
        if (p.P != nullptr && cta == 0 && row < rows && j < r) p.P[(size_t)(m0 + row) * r + j] = v;
        sh.low[row][j] = e >= 0 && p.scales != nullptr ? p.scales[sh.entry_adapter[e]] * v : 0.f;
    }
    __syncthreads();
    if constexpr (FORWARD) {
        // ---- the second product with B [C, r]: NT threads share a column, eight ranks each, so that a warp reads in one stretch
        constexpr int BATCH = 8;
        const int j = lane % NT, c_lo = 2 * p_lo, total = 2 * (p_hi - p_lo) * NT;
        float low[ROWS][8];
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) low[i][k] = sh.low[i][8 * j + k];
        for (int e = 0; e < n_entries; ++e) {
            const bf16* La = p.L2 + (size_t)sh.entry_adapter[e] * r * C + 8 * j;
            const uint32_t mask = sh.entry_mask[e];
            for (int at = warp * 32; at < total; at += THREADS * BATCH) {
                uint4 w[BATCH];
                uint32_t base[BATCH][ROWS];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    const int i = at + u * THREADS + lane, c = c_lo + i / NT;
                    w[u] = i < total && 8 * j < r ? ldg16(La + (size_t)c * r) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < ROWS; ++k)
                        base[u][k] = j == 0 && i < total && ((mask >> k) & 1u) ? *reinterpret_cast<const uint16_t*>(p.Base + (size_t)(m0 + k) * C + c) : 0u;
                }
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    const int i = at + u * THREADS + lane, c = c_lo + i / NT;
                    const uint32_t v[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        float s = 0.f;
#pragma unroll
                        for (int h = 0; h < 4; ++h) s = fmaf(low[k][2 * h], bf16_lo(v[h]), fmaf(low[k][2 * h + 1], bf16_hi(v[h]), s));
#pragma unroll
                        for (int o = 1; o < NT; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
                        if (j == 0 && i < total && ((mask >> k) & 1u)) p.Out[(size_t)(m0 + k) * C + c] = __float2bfloat16_rn(bf16_lo(base[u][k]) + s);
                    }
                }
            }
        }
    } else {
        // ---- the second product with A [r, C]: a thread has two neighbouring columns of one entry, BATCH such units at a time
        constexpr int BATCH = NT <= 2 ? 4 : NT <= 4 ? 2 : 1;
        const int n_pairs = p_hi - p_lo, units = n_entries * n_pairs;
        for (int unit0 = threadIdx.x; unit0 < units; unit0 += THREADS * BATCH) {
            uint32_t w[BATCH][NT * 8], base[BATCH][ROWS], masks[BATCH];
            int column[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int unit = unit0 + u * THREADS, e = ROWS > 1 && unit < units ? unit / n_pairs : 0, c = 2 * (p_lo + (unit < units ? unit - e * n_pairs : 0));
                column[u] = c;
                masks[u] = unit < units ? sh.entry_mask[e] : 0u;
                const bf16* La = p.L2 + (size_t)sh.entry_adapter[e] * r * C;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (8 * j >= r) break;
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[u][8 * j + i] = __ldg(reinterpret_cast<const uint32_t*>(La + (size_t)(8 * j + i) * C + c));
                }
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    base[u][i] = (masks[u] >> i) & 1u ? *reinterpret_cast<const uint32_t*>(p.Base + (size_t)(m0 + i) * C + c) : 0u;
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u)
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    if (!((masks[u] >> i) & 1u)) continue;
                    float a = 0.f, b = 0.f;
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        if (8 * j >= r) break;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float v = sh.low[i][8 * j + k];
                            a = fmaf(v, bf16_lo(w[u][8 * j + k]), a);
                            b = fmaf(v, bf16_hi(w[u][8 * j + k]), b);
                        }
                    }
                    *reinterpret_cast<uint32_t*>(p.Out + (size_t)(m0 + i) * C + column[u]) = bf16x2(bf16_lo(base[u][i]) + a, bf16_hi(base[u][i]) + b);
                }
        }
    }
    if (p.Out != p.Base)                                               // tokens without an adapter
        for (int i = 0; i < rows; ++i)
            if (sh.entry_of[i] < 0)
                for (int c = p_lo + threadIdx.x; c < p_hi; c += THREADS)
                    *reinterpret_cast<uint32_t*>(p.Out + (size_t)(m0 + i) * C + 2 * c) = *reinterpret_cast<const uint32_t*>(p.Base + (size_t)(m0 + i) * C + 2 * c);
}

template <bool FORWARD, int NT, int ROWS, int CTAS>
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(32 * FEW_WARPS, 2)
adapters_few_kernel(const Products p) {
    __shared__ __align__(16) FewShared<NT, ROWS, CTAS> sh;
    pdl_launch_dependents();
    cluster_arrive();                                                  // (a CTA's shared memory is written to once it has begun)
    pdl_wait();
    cluster_wait();
    few_tokens<FORWARD, NT, ROWS, CTAS>(p, (int)(blockIdx.x / CTAS) * ROWS, sh);
}

// ---------------------------------------------------------------------------------------------------------------- down
// Many tokens, the first product.  A block has 16 NB tokens and reads their rows of In once where they have one adapter; its warps stride over the
// contraction (fragments as in lora_down.cuh) and add their sums in order.  The second product gets s P as two bf16 each from here, so that it
// need not take every value apart again for each of its columns.  Bound by DRAM latency and what is under way: 34.6 MB in 14 us (4096 tokens, 4096 long, rank 16),
// 92 MB in 24 us (11008 long, rank 8).
//
// Tiles of 16 tokens with more than two adapters (short requests, single tokens in generation beside the prompts of others) would be up to sixteen tiles' work for one
// block, and would read an adapter again for every tile that one of its tokens is in.  Their tokens are sorted by adapter by a block beside the other tiles' work, and
// are worked on in groups of up to sixteen: by helpers, blocks without a tile, and by those whose own tile is such a one, which claim group by group.
// (4096 x 4096, rank 16, both products: 1024 tokens of 32 adapters in turn 30 us, token by token it was 290; 8192 of them 141 us, was 2640.  A batch without such a
// tile pays 1.5 us for the sorting kernel's launch.)
constexpr int DN_WARPS = 8, DN_ENTRIES = 2, DN_HELPERS = 32;

// Lane i holds the adapter of token i of one (16 lanes) or two tiles: whether its tile is one of more than DN_ENTRIES adapters.
__device__ __forceinline__ bool of_scattered_tile(int adapter) {
    const int lane = threadIdx.x & 31;
    const uint32_t half = lane < 16 ? 0x0000FFFFu : 0xFFFF0000u, same = __match_any_sync(0xFFFFFFFFu, adapter) & half;
    const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, adapter >= 0 && (same & ((1u << lane) - 1u)) == 0) & half;
    return __popc(firsts) > DN_ENTRIES;
}

// One block; 4096 tokens at a time are sorted (bitonic, 78 steps at most, fewer where fewer are to be sorted).  Tokens of such tiles without an adapter are groups as
// well.  The next kernel is let in once this one has waited for what was before: its tiles need nothing from here, so they do not wait.
constexpr int SORT_THREADS = 1024, SORT_ROUNDS = 4, SORT_WINDOW = SORT_THREADS * SORT_ROUNDS;
__global__ void __launch_bounds__(SORT_THREADS)
adapters_groups_kernel(int M, int n_adapters, const int32_t* __restrict__ adapter_of, const Groups out) {
    __shared__ uint32_t keys[SORT_WINDOW];                             // adapter << 12 | token of the window
    __shared__ int counts[SORT_ROUNDS * 32], total_s;
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // how many of the flags of all rounds come before this thread's
    auto places = [&](const bool (&flag)[SORT_ROUNDS], int (&at)[SORT_ROUNDS]) {
        uint32_t votes[SORT_ROUNDS];
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) {
            votes[k] = __ballot_sync(0xFFFFFFFFu, flag[k]);
            if (lane == 0) counts[k * 32 + warp] = __popc(votes[k]);
        }
        __syncthreads();
        if (warp == 0) {
            int mine[SORT_ROUNDS], sum = 0;
#pragma unroll
            for (int k = 0; k < SORT_ROUNDS; ++k) { mine[k] = sum; sum += counts[lane * SORT_ROUNDS + k]; }
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane >= o) before += x;
            }
            if (lane == 31) total_s = before;
#pragma unroll
            for (int k = 0; k < SORT_ROUNDS; ++k) counts[lane * SORT_ROUNDS + k] = before - sum + mine[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) at[k] = counts[k * 32 + warp] + __popc(votes[k] & ((1u << lane) - 1u));
        const int total = total_s;
        __syncthreads();
        return total;
    };
    int n_tokens = 0, n_groups = 0;
    for (int w0 = 0; w0 < M; w0 += SORT_WINDOW) {
        int a[SORT_ROUNDS], at[SORT_ROUNDS];
        bool flag[SORT_ROUNDS], any = false;
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) {
            const int t = w0 + k * SORT_THREADS + threadIdx.x;
            a[k] = t < M ? __ldg(adapter_of + t) : -1;
        }
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) {
            if (a[k] < 0 || a[k] >= n_adapters) a[k] = -1;
            flag[k] = of_scattered_tile(a[k]) && w0 + k * SORT_THREADS + (int)threadIdx.x < M;
            any |= flag[k];
        }
        if (!__syncthreads_or(any)) continue;
        const int n = places(flag, at);
        int size = 32;
        while (size < n) size *= 2;
        for (int i = n + threadIdx.x; i < size; i += SORT_THREADS) keys[i] = 0xFFFFFFFFu;
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k)
            if (flag[k]) keys[at[k]] = (uint32_t)(a[k] < 0 ? NO_ADAPTER : a[k]) << 12 | (uint32_t)(k * SORT_THREADS + threadIdx.x);
        __syncthreads();
        for (int run = 2; run <= size; run *= 2)
            for (int apart = run / 2; apart > 0; apart /= 2) {
                for (int i = threadIdx.x; i < size / 2; i += SORT_THREADS) {
                    const int lo = 2 * i - (i & (apart - 1)), hi = lo + apart;
                    const uint32_t x = keys[lo], y = keys[hi];
                    if ((x > y) == ((lo & run) == 0)) { keys[lo] = y; keys[hi] = x; }
                }
                __syncthreads();
            }
        auto first_of = [&](uint32_t key) {                            // the first place whose key is not below
            int lo = 0, hi = n;
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (keys[mid] < key) lo = mid + 1;
                else hi = mid;
            }
            return lo;
        };
        int many[SORT_ROUNDS];
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) {
            const int j = k * SORT_THREADS + threadIdx.x;
            flag[k] = false;
            many[k] = 0;
            if (j >= n) continue;
            const uint32_t adapter = keys[j] >> 12;
            flag[k] = (j - first_of(adapter << 12)) % GROUP == 0;
            if (flag[k]) many[k] = min(GROUP, first_of((adapter + 1) << 12) - j);
            out.tokens[n_tokens + j] = w0 + (int)(keys[j] & (SORT_WINDOW - 1));
        }
        const int more = places(flag, at);
#pragma unroll
        for (int k = 0; k < SORT_ROUNDS; ++k) {
            const int j = k * SORT_THREADS + threadIdx.x;
            if (flag[k]) out.groups[n_groups + at[k]] = make_int2((n_tokens + j) << 5 | many[k], (int)(keys[j] >> 12));
        }
        n_tokens += n;
        n_groups += more;
        __syncthreads();
    }
    if (threadIdx.x == 0) { out.head[0] = n_groups; out.head[1] = 0; }
}

// Every warp has a ring of its own in shared memory, a stage of which holds 64 contraction elements of the tile's rows and of the adapter; copies
// run ahead without holding registers.  16-byte pieces are XORed by row, so that the matrix loads have no bank conflicts.  Where there are few tiles a
// cluster of CTAS blocks shares the contraction out, and its first one adds their sums in order.
template <bool L_IS_A, int NT, int NB, int CTAS>
struct DownTile {
    static constexpr int ROWS = 16 * NB, CHUNK = 64;
    static constexpr int IN_BYTES = ROWS * 128, L_BYTES = NT * 8 * 128, STAGE = IN_BYTES + L_BYTES;
    static constexpr int STAGES = NT == 1 ? 4 : NT == 2 ? 3 : 2;
    static constexpr size_t RING = (size_t)STAGES * STAGE * DN_WARPS, SUMS = sizeof(float) * DN_WARPS * NB * NT * 128;
    static constexpr size_t OWN = RING > SUMS ? RING : SUMS, PARTS = CTAS > 1 ? CTAS * NB * NT * 64 * sizeof(float2) : 0;
    static constexpr size_t SMEM = OWN + PARTS;
};

template <bool L_IS_A, int NT, int NB, int CTAS>
__global__ void __launch_bounds__(32 * DN_WARPS, NT <= 4 ? 2 : 1)
adapters_down_kernel(const Products p, int n_tiles) {
    using Tile = DownTile<L_IS_A, NT, NB, CTAS>;
    constexpr int ROWS = Tile::ROWS, CHUNK = Tile::CHUNK, STAGES = Tile::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    auto& red = *reinterpret_cast<float (*)[DN_WARPS][NB][NT][4][32]>(smem);
    __shared__ int claimed, tokens[ROWS];                              // of a group: the number of a row's token, -1 for none
    // No wait ahead of the tiles: the sorting kernel lets this one begin after its own wait, when all kernels before it have completed and their writes lie in L2, which is
    // where the tiles read everything from (asynchronous copies and loads past L1).  What the sorting kernel itself writes is waited for below.
    pdl_launch_dependents();
    if (CTAS > 1) cluster_sync_all();                                  // (a block's shared memory is written to once it has begun)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int M = p.M, T = p.T, r = p.r;
    const int m0 = (int)blockIdx.x / CTAS * ROWS, cta = CTAS > 1 ? (int)cluster_ctarank() : 0;
    constexpr int ALL = DN_WARPS * CTAS;                               // warps of the tile
    const int me = cta * DN_WARPS + warp;
    const uint32_t ring = smem_u32(smem) + warp * STAGES * Tile::STAGE;
    const int chunks = (T + CHUNK - 1) / CHUNK, mine = me < chunks ? (chunks - me + ALL - 1) / ALL : 0;
    // what a lane copies: a 16-byte piece of every fourth row of the tile, and of the adapter
    const int piece = lane & 7, row0 = lane >> 3;
    const bf16* in0 = p.In + (size_t)(m0 + row0) * T + me * CHUNK + 8 * piece;
    uint32_t rows_in = 0;
#pragma unroll
    for (int n = 0; n < ROWS / 4; ++n) rows_in |= (uint32_t)(m0 + row0 + 4 * n < M) << n;
    const std::false_type of_tile{};
    const std::true_type of_group{};
    const uint32_t swizzled[2] = {(uint32_t)(row0 * 128 + ((piece ^ row0) << 4)), (uint32_t)(row0 * 128 + ((piece ^ (row0 + 4)) << 4))};   // rows 4 n: n even, odd
    auto load_in = [&](int i, auto gathered) {                         // chunk i of this warp's
        const int from = i * (ALL * CHUNK);
        const bool k_in = me * CHUNK + 8 * piece + from < T;
        const bf16* src = in0 + from;
        const uint32_t to = ring + (i % STAGES) * Tile::STAGE;
#pragma unroll
        for (int n = 0; n < ROWS / 4; ++n) {
            if constexpr (gathered.value) {
                const int t = tokens[row0 + 4 * n];
                const bool in = k_in && t >= 0;
                copy16(to + 512 * n + swizzled[n & 1], in ? p.In + (size_t)t * T + me * CHUNK + 8 * piece + from : p.In, in);
            } else {
                const bool in = k_in && ((rows_in >> n) & 1u);
                copy16(to + 512 * n + swizzled[n & 1], in ? src : p.In, in);
                src += (size_t)4 * T;
            }
        }
    };
    auto load_adapter = [&](int i, const bf16* La) {
        const int from = i * (ALL * CHUNK), k0 = me * CHUNK + from;
        const uint32_t to = ring + (i % STAGES) * Tile::STAGE + Tile::IN_BYTES;
        if constexpr (L_IS_A) {                                        // rows of ranks, 64 elements each
            const bool k_in = k0 + 8 * piece < T;
            const bf16* src = La + (size_t)row0 * T + k0 + 8 * piece;
#pragma unroll
            for (int n = 0; n < 2 * NT; ++n) {
                const bool in = k_in && 4 * n + row0 < r;
                copy16(to + 512 * n + swizzled[n & 1], in ? src : La, in);
                src += (size_t)4 * T;
            }
        } else {                                                       // rows of contraction elements, 8 NT ranks each
#pragma unroll
            for (int n = 0; n < 2 * NT; ++n) {
                const int at = 32 * n + lane, k = at / NT, j = at % NT;
                const bool in = k0 + k < T && 8 * j < r;
                copy16(to + k * (16 * NT) + ((j ^ ((k * NT / 8) % NT)) << 4), La + (in ? (size_t)(k0 + k) * r + 8 * j : 0), in);
            }
        }
    };
    const uint32_t parts = smem_u32(smem) + (uint32_t)Tile::OWN;
    // The sums of one adapter's rows (mask) of the tile, or of a group.  begun: the first chunks of In are on their way.
    auto entry = [&](auto gathered, int adapter, uint32_t mask, bool begun) {
        const bf16* La = p.L1 + (size_t)adapter * r * T;
        const float s = p.scales != nullptr ? __ldcg(p.scales + adapter) : 0.f;
        // two neighbouring ranks of a row
        auto take = [&](int idx, float v0, float v1) {
            const int b = idx / (NT * 64), nt = (idx >> 6) % NT, h = (idx >> 5) & 1, ln = idx & 31;
            const int row = 16 * b + (ln >> 2) + 8 * h, col = nt * 8 + (ln & 3) * 2;
            if (!((mask >> row) & 1u) || col >= r) return;
            const size_t token = gathered.value ? tokens[row] : m0 + row;
            if (p.P != nullptr) *reinterpret_cast<float2*>(p.P + token * r + col) = make_float2(v0, v1);
            if (p.split != nullptr) {
                const Split v = split_bf16(s * v0, s * v1);
                uint2* to = p.split + token * split_pairs(r) + (L_IS_A ? col / 2 : col / 16 * 8 + col % 8 + col / 8 % 2);
                to[0] = make_uint2(v.hi, v.lo);
                if (!L_IS_A && r % 16 == 8 && col >= r - 8) to[1] = make_uint2(0u, 0u);      // the ranks that there are not
            }
        };
        float acc[NB][NT][4] = {};
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) {
            if (i < mine) {
                if (!begun) load_in(i, gathered);
                load_adapter(i, La);
            }
            copy_commit();
        }
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            copy_wait<STAGES - 2>();
            __syncwarp();                                              // chunk i is there, chunk i - 1 has been read by every lane
            if (i + STAGES - 1 < mine) {
                load_in(i + STAGES - 1, gathered);
                load_adapter(i + STAGES - 1, La);
            }
            copy_commit();
            const uint32_t x = ring + (i % STAGES) * Tile::STAGE, l = x + Tile::IN_BYTES;
            const int row8 = lane & 7, quarter = lane >> 3;            // matrix `quarter` of four, its row `row8`
#pragma unroll
            for (int k = 0; k < CHUNK / 16; ++k) {
                uint32_t xa[NB][4];
#pragma unroll
                for (int b = 0; b < NB; ++b) {                         // rows 0 - 7, 8 - 15 of elements 0 - 7; then of 8 - 15
                    const int row = 16 * b + row8 + 8 * (quarter & 1), piece = 2 * k + (quarter >> 1);
                    ldmatrix4<false>(x + row * 128 + ((piece ^ (row & 7)) << 4), xa[b][0], xa[b][1], xa[b][2], xa[b][3]);
                }
                uint32_t lb[NT][2];
                if constexpr (NT == 1) {                               // (two steps' worth is not worth the registers: the second half of the four is not used)
                    uint32_t u0, u1;
                    if constexpr (L_IS_A) ldmatrix4<false>(l + row8 * 128 + (((2 * k + (quarter & 1)) ^ row8) << 4), lb[0][0], lb[0][1], u0, u1);
                    else ldmatrix4<true>(l + (16 * k + row8 + 8 * (quarter & 1)) * 16, lb[0][0], lb[0][1], u0, u1);
                } else {
#pragma unroll
                    for (int nt = 0; nt < NT; nt += 2) {
                        if constexpr (L_IS_A) {
                            const int j = 8 * (nt + (quarter >> 1)) + row8, piece = 2 * k + (quarter & 1);
                            ldmatrix4<false>(l + j * 128 + ((piece ^ row8) << 4), lb[nt][0], lb[nt][1], lb[nt + 1][0], lb[nt + 1][1]);
                        } else {
                            const int e = 16 * k + row8 + 8 * (quarter & 1), j = nt + (quarter >> 1);
                            ldmatrix4<true>(l + e * (16 * NT) + ((j ^ ((e * NT / 8) % NT)) << 4), lb[nt][0], lb[nt][1], lb[nt + 1][0], lb[nt + 1][1]);
                        }
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(acc[b][nt], xa[b][0], xa[b][1], xa[b][2], xa[b][3], lb[nt][0], lb[nt][1]);
            }
        }
        copy_wait<0>();
        __syncthreads();                                               // the sums lie where the rings are
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) red[warp][b][nt][c][lane] = acc[b][nt][c];
        __syncthreads();
        for (int idx = threadIdx.x; idx < NB * NT * 64; idx += 32 * DN_WARPS) {
            const int b = idx / (NT * 64), nt = (idx >> 6) % NT, h = (idx >> 5) & 1, ln = idx & 31;
            float v0 = 0.f, v1 = 0.f;
#pragma unroll
            for (int w = 0; w < DN_WARPS; ++w) { v0 += red[w][b][nt][2 * h][ln]; v1 += red[w][b][nt][2 * h + 1][ln]; }
            if constexpr (CTAS > 1) {
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(map_to_cta(parts + 8 * (cta * NB * NT * 64 + idx), 0)), "f"(v0), "f"(v1) : "memory");
                continue;
            }
            take(idx, v0, v1);
        }
        if constexpr (CTAS > 1) {
            __syncwarp();
            cluster_sync_all();
            if (cta == 0)
                for (int idx = threadIdx.x; idx < NB * NT * 64; idx += 32 * DN_WARPS) {
                    float2 v = make_float2(0.f, 0.f);
#pragma unroll
                    for (int i = 0; i < CTAS; ++i) {
                        const float2 x = *reinterpret_cast<const float2*>(smem + Tile::OWN + 8 * (i * NB * NT * 64 + idx));
                        v.x += x.x;
                        v.y += x.y;
                    }
                    take(idx, v.x, v.y);
                }
            __syncwarp();
            cluster_sync_all();                                        // (the next entry's sums go where these were)
        }
        __syncthreads();
    };
    if ((int)blockIdx.x < n_tiles) {
        const bool in = lane < ROWS && m0 + lane < M;
        int a = in ? __ldcg(p.adapter_of + m0 + lane) : -1;
        for (int i = 0; i < STAGES - 1 && i < mine; ++i) load_in(i, of_tile);      // on their way while the tile's adapters are looked at
        if (a < 0 || a >= p.n_adapters) a = -1;
        const bool elsewhere = of_scattered_tile(a);
        if (me == 0 && p.P != nullptr && in && a < 0 && !elsewhere)
            for (int j = 0; j < r; j += 4) *reinterpret_cast<float4*>(p.P + (size_t)(m0 + lane) * r + j) = make_float4(0.f, 0.f, 0.f, 0.f);
        if (elsewhere) a = -1;
        const uint32_t mask_here = entry_of_lane(a);
        uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mask_here != 0);
        for (bool begun = true; firsts != 0; firsts &= firsts - 1, begun = false) {
            const int first = __ffs(firsts) - 1;
            entry(of_tile, __shfl_sync(0xFFFFFFFFu, a, first), __shfl_sync(0xFFFFFFFFu, mask_here, first), begun);
        }
        copy_commit();
        copy_wait<0>();                                                // (a tile without an entry leaves with its copies done)
        if (!__any_sync(0xFFFFFFFFu, elsewhere)) return;               // (the same for all warps)
    }
    pdl_wait();
    const int n_groups = __ldcg(p.groups.head);
    for (;;) {
        if constexpr (CTAS > 1) cluster_sync_all();
        else __syncthreads();                                          // what was claimed before has been read
        if (cta == 0 && threadIdx.x == 0) {
            claimed = atomicAdd(p.groups.head + 1, 1);
            if constexpr (CTAS > 1)
                for (int i = 1; i < CTAS; ++i) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(&claimed), i)), "r"(claimed) : "memory");
        }
        __syncwarp();
        if constexpr (CTAS > 1) cluster_sync_all();
        else __syncthreads();
        if (claimed >= n_groups) return;
        const int2 group = __ldcg(p.groups.groups + claimed);
        const int many = group.x & 31;
        if (threadIdx.x < ROWS) tokens[threadIdx.x] = (int)threadIdx.x < many ? __ldcg(p.groups.tokens + (group.x >> 5) + threadIdx.x) : -1;
        __syncthreads();
        if (group.y != NO_ADAPTER) entry(of_group, group.y, (1u << many) - 1u, false);
        else if (cta == 0 && p.P != nullptr)
            for (int i = threadIdx.x; i < many * r; i += 32 * DN_WARPS) p.P[(size_t)tokens[i / r] * r + i % r] = 0.f;
    }
}

// ------------------------------------------------------------------------------------------------------------------ up
// Many tokens, the second product.  A warp has 32 UB columns and goes down the rows, sixteen at a time.  It keeps its columns of the adapter in registers
// for as long as the adapter stays the same, so long requests read Base and write Out and little else; the next rows are asked for a tile ahead.
// Bound by DRAM: 184 MB in 35 us, 5.3 TB/s (4096 tokens, 11008 columns, rank 16).
constexpr int UP_ROWS = 16, UP_WARPS = 8;

// Ranks 16 ks .. 16 ks + 15 of 32 columns (c0 ..) as four column tiles of an MMA.  Column c of tile t is c0 + 8 (c / 2) + 2 t + c % 2, so that a
// thread's sums are eight neighbouring columns.  FROM_B: L2 = B [C, r]; else A [r, C].  The ranks are in the order (4 q, 4 q + 1; 4 q + 2, 4 q + 3) for B,
// which is read along them, and (2 q, 2 q + 1; 8 + 2 q, 9 + 2 q) for A.
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

// What lane q takes of the ranks 16 ks .. 16 ks + 15 of token t's s P, in that order, each pair (high, low).  (With eight ranks left the others' places hold zeros.)
template <bool FROM_B>
__device__ __forceinline__ uint4 up_low(const Products& p, int t, int ks, int q) {
    const bool in = FROM_B ? 16 * ks + 4 * q < p.r : 16 * ks < p.r;
    return in ? *reinterpret_cast<const uint4*>(p.split + (size_t)t * split_pairs(p.r) + 8 * ks + 2 * q) : make_uint4(0, 0, 0, 0);
}

// A group of tokens, a warp's columns of them.
template <bool FROM_B, int KS, int UB>
__device__ __forceinline__ void up_group(const Products& p, int group, int c_warp) {
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, C = p.C, r = p.r;
    if (c_warp >= C) return;
    const int2 what = __ldcg(p.groups.groups + group);
    const int many = what.x & 31;
    int token[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) token[h] = g + 8 * h < many ? __ldcg(p.groups.tokens + (what.x >> 5) + g + 8 * h) : -1;
    const bool none = what.y == NO_ADAPTER;
    if (none && p.Out == p.Base) return;
    uint4 base[UB][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < UB; ++i) {
            const int c = c_warp + 32 * i + 8 * q;
            base[i][h] = token[h] >= 0 && c < C ? *reinterpret_cast<const uint4*>(p.Base + (size_t)token[h] * C + c) : make_uint4(0, 0, 0, 0);
        }
    if (!none) {
        float sum[UB][4][4];
#pragma unroll
        for (int i = 0; i < UB; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w[4] = {base[i][h].x, base[i][h].y, base[i][h].z, base[i][h].w};
#pragma unroll
                for (int t = 0; t < 4; ++t) { sum[i][t][2 * h] = bf16_lo(w[t]); sum[i][t][2 * h + 1] = bf16_hi(w[t]); }
            }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 low[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) low[h] = token[h] >= 0 ? up_low<FROM_B>(p, token[h], ks, q) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < UB; ++i) {
                uint32_t b[4][2];
                up_fragments<FROM_B>(p.L2 + (size_t)what.y * r * C, C, r, c_warp + 32 * i, ks, g, q, b);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    mma_bf16_16816(sum[i][t], low[0].x, low[1].x, low[0].z, low[1].z, b[t][0], b[t][1]);
                    mma_bf16_16816(sum[i][t], low[0].y, low[1].y, low[0].w, low[1].w, finite_pair(b[t][0]), finite_pair(b[t][1]));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < UB; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                base[i][h] = make_uint4(bf16x2(sum[i][0][2 * h], sum[i][0][2 * h + 1]), bf16x2(sum[i][1][2 * h], sum[i][1][2 * h + 1]),
                                        bf16x2(sum[i][2][2 * h], sum[i][2][2 * h + 1]), bf16x2(sum[i][3][2 * h], sum[i][3][2 * h + 1]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < UB; ++i) {
            const int c = c_warp + 32 * i + 8 * q;
            if (token[h] >= 0 && c < C) *reinterpret_cast<uint4*>(p.Out + (size_t)token[h] * C + c) = base[i][h];
        }
}

// KS steps of 16 ranks.  A warp has 64 columns, so that a row of s P is loaded for every 64; above one step that takes the registers of one block an SM (8192 tokens, 4096
// x 4096, both products, forward and backward: rank 32 68 -> 65 and 84 -> 66 us against 32 columns and two blocks, rank 64 93 -> 88 and 115 -> 91).
constexpr int up_blocks(int steps) { return steps > 1 ? 1 : 2; }
template <bool FROM_B, int KS, int UB>
__global__ void __launch_bounds__(32 * UP_WARPS, up_blocks(KS))
adapters_up_kernel(const Products p, int tiles_each) {
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int c_warp = (blockIdx.y * UP_WARPS + warp) * 32 * UB, M = p.M, C = p.C, r = p.r;
    const int n_groups = __ldcg(p.groups.head);
    const int tiles = (M + UP_ROWS - 1) / UP_ROWS, tile_end = c_warp < C ? min(tiles, ((int)blockIdx.x + 1) * tiles_each) : 0;
    struct Tile {
        uint4 base[UB][2];
        int adapter;                                                   // of row `lane`, modulo sixteen
    };
    struct Low { uint4 v[KS][2]; };                                    // [step][row]: both halves of the step's ranks, each (high, low)
    int tile = blockIdx.x * tiles_each;
    const size_t at0 = (size_t)(tile * UP_ROWS + g) * C + c_warp + 8 * q;      // this lane's first element
    bool c_in[UB];
#pragma unroll
    for (int i = 0; i < UB; ++i) c_in[i] = c_warp + 32 * i + 8 * q < C;
    // (`ahead`: how many tiles this one lies behind the block's first; `whole`: all its rows exist)
    auto load = [&](int ahead, bool whole, Tile& x) {
        const int m0 = (tile + ahead) * UP_ROWS, row = m0 + (lane & 15);
        x.adapter = whole || row < M ? __ldg(p.adapter_of + row) : -1;
        const bf16* from = p.Base + at0 + (size_t)(m0 - (int)blockIdx.x * tiles_each * UP_ROWS) * C;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < UB; ++i)
                x.base[i][h] = c_in[i] && (whole || m0 + g + 8 * h < M) ? *reinterpret_cast<const uint4*>(from + (size_t)(8 * h) * C + 32 * i) : make_uint4(0, 0, 0, 0);
    };
    auto load_low = [&](int ahead, bool whole, Low& x) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = (tile + ahead) * UP_ROWS + g + 8 * h;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                x.v[ks][h] = whole || row < M ? up_low<FROM_B>(p, row, ks, q) : make_uint4(0, 0, 0, 0);
        }
    };
    uint32_t held[KS][UB][4][2];
    int held_adapter = -1;
    bool held_finite = true;
    Tile x;
    Low low;
    auto whole = [&](int i) { return (i + 1) * UP_ROWS <= M; };
    if (tile < tile_end) {
        load(0, whole(tile), x);
        load_low(0, whole(tile), low);
    }
#pragma unroll 1
    for (; tile < tile_end; ++tile) {
        Tile following;
        Low following_low;
        if (tile + 1 < tile_end) {
            load(1, whole(tile + 1), following);
            load_low(1, whole(tile + 1), following_low);
        }
        const int m0 = tile * UP_ROWS;
        const int a = x.adapter >= 0 && x.adapter < p.n_adapters ? x.adapter : -1;
        uint32_t mask_here = 0xFFFFu, firsts = 1u;
        bool elsewhere = false;                                        // one of the tiles that are left for the end
        const bool one = held_adapter >= 0 && __all_sync(0xFFFFFFFFu, a == held_adapter);   // the adapter before, in every row
        if (!one) {
            mask_here = entry_of_lane(lane < UP_ROWS ? a : -1);
            firsts = __ballot_sync(0xFFFFFFFFu, mask_here != 0);
            elsewhere = __popc(firsts) > DN_ENTRIES;
            if (elsewhere) firsts = 0;
        }
        while (firsts != 0) {
            const int first = __ffs(firsts) - 1;
            firsts &= firsts - 1;
            const uint32_t mask = one ? 0xFFFFu : __shfl_sync(0xFFFFFFFFu, mask_here, first);
            const int adapter = one ? held_adapter : __shfl_sync(0xFFFFFFFFu, a, first);
            if (adapter != held_adapter) {                             // (the same for the whole warp)
                const bf16* L2 = p.L2 + (size_t)adapter * r * C;
                uint32_t odd = 0;                                      // bits 15 and 31: an exponent of all ones
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int i = 0; i < UB; ++i) {
                        up_fragments<FROM_B>(L2, C, r, c_warp + 32 * i, ks, g, q, held[ks][i]);
#pragma unroll
                        for (int t = 0; t < 4; ++t) odd |= ((held[ks][i][t][0] & 0x7F807F80u) + 0x00800080u) | ((held[ks][i][t][1] & 0x7F807F80u) + 0x00800080u);
                    }
                held_finite = !__any_sync(0xFFFFFFFFu, (odd & 0x80008000u) != 0);
                held_adapter = adapter;
            }
            // the rows of Base and on top of them the products with both parts of s P.  (A row of the result depends on its own row of P alone: rows of other
            // entries are computed and not stored.)
            float sum[UB][4][4];
#pragma unroll
            for (int i = 0; i < UB; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w[4] = {x.base[i][h].x, x.base[i][h].y, x.base[i][h].z, x.base[i][h].w};
#pragma unroll
                    for (int t = 0; t < 4; ++t) { sum[i][t][2 * h] = bf16_lo(w[t]); sum[i][t][2 * h + 1] = bf16_hi(w[t]); }
                }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const uint4 v0 = low.v[ks][0], v1 = low.v[ks][1];
#pragma unroll
                for (int i = 0; i < UB; ++i)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t b0 = held[ks][i][t][0], b1 = held[ks][i][t][1];
                        mma_bf16_16816(sum[i][t], v0.x, v1.x, v0.z, v1.z, b0, b1);
                        if (held_finite) mma_bf16_16816(sum[i][t], v0.y, v1.y, v0.w, v1.w, b0, b1);
                        else mma_bf16_16816(sum[i][t], v0.y, v1.y, v0.w, v1.w, finite_pair(b0), finite_pair(b1));
                    }
            }
            bf16* to = p.Out + (size_t)(m0 + g) * C + c_warp + 8 * q;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!((mask >> (g + 8 * h)) & 1u)) continue;
#pragma unroll
                for (int i = 0; i < UB; ++i)
                    if (c_in[i])
                        *reinterpret_cast<uint4*>(to + (size_t)(8 * h) * C + 32 * i) =
                            make_uint4(bf16x2(sum[i][0][2 * h], sum[i][0][2 * h + 1]), bf16x2(sum[i][1][2 * h], sum[i][1][2 * h + 1]),
                                       bf16x2(sum[i][2][2 * h], sum[i][2][2 * h + 1]), bf16x2(sum[i][3][2 * h], sum[i][3][2 * h + 1]));
            }
        }
        if (!one && !elsewhere && p.Out != p.Base) {                   // tokens without an adapter keep their bits, whatever they are
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = m0 + g + 8 * h;
                if (__shfl_sync(0xFFFFFFFFu, a, g + 8 * h) >= 0 || row >= M) continue;
#pragma unroll
                for (int i = 0; i < UB; ++i)
                    if (c_in[i]) *reinterpret_cast<uint4*>(p.Out + (size_t)row * C + c_warp + 32 * i + 8 * q) = x.base[i][h];
            }
        }
        x = following;
        low = following_low;
    }
    // the groups, a block's columns at a time, all blocks in turn
    const int slabs = gridDim.y;
#pragma unroll 1
    for (int i = blockIdx.y * gridDim.x + blockIdx.x; i < n_groups * slabs; i += gridDim.x * slabs)
        up_group<FROM_B, KS, UB>(p, i / slabs, (i % slabs * UP_WARPS + warp) * 32 * UB);
}

// --------------------------------------------------------------------------------------------------------------- grads
// First the tiles of sixteen tokens are listed with the adapters in them (an entry: adapter, tile, mask of its tokens), in the order of the tokens, and every
// adapter's entries are cut into chunks of equal length: adapters differ in their tokens, and the one with the most would be what all wait for.  A task is
// a chunk, a slice of columns of X or of dY (128 up to 16 ranks, else 64) and 16 MT ranks; blocks claim tasks one by one, slices first, so that those under
// way at a time read whole rows.  A block picks its chunk's entries out of the list; its warps take them in turn, each through a ring of its own in shared
// memory, rows of other adapters as zeros, and their sums are added in the order of the warps.  The block that finishes an adapter's last chunk of a
// slice adds the chunks in their order.
//
// Bound by the tasks' own ends (the first loads, the sums of four warps, the chunks' sums) and the chain of a warp's instructions, not by the bytes: 68 MB in 31 us after
// 10 us of listing (4096 tokens, 4096 x 4096, rank 16, three blocks an SM: 12 warps, an instruction every 8.6 cycles each).  In all 37.7 us; chunks of 40 tiles at least 40.0, but 39
// instead of 41 for 1531 tokens of 13 sequences; 8 warps, or two blocks with four stages, were slower or no faster, and so were 128 columns above rank 16 (231 -> 249).
//
// Both operands are transposed on the way out of shared memory.  G and H are taken as three bf16 each, which hold all of an fp32 value (made once, not by every
// slice; with two the gradients were 2.5e-6 off, with three 5e-7), one product after the other into the same sums.  Where a sum is not finite the lower parts
// may have made a NaN of an infinity in X or dY: the task is then done again with zeros for them there, and finite sums come out as before.
constexpr int GR_PARTS = 3, GR_WARPS = 4, GR_STAGES = 3, GR_BLOCKS = 3, GR_MIN_TILES = 32;

struct Grads {
    int M, K, N, r, n_adapters;
    const bf16 *X, *dY;                      // [M, K], [M, N]
    const int32_t* adapter_of;
    const float* scales;
    const bf16 *G, *H;                       // [GR_PARTS][M, r]: from the highest parts down
    float *dA, *dB;
    int accumulate;
    int slices_x, slices, rank_blocks;
    int most_chunks;                         // chunks of adapters that have more than one: at most twice as many
    unsigned* counters;                      // [0] claimed, [1] entries, [2] tiles of a chunk, [3] chunks; [4 ..] chunks done, by first chunk of an adapter of several and slice
    uint2* entries;                          // [M]: adapter, tile << 16 | mask (tile < 65536: up to 2^20 tokens)
    int* counts;                             // [n_adapters]: entries
    int4* chunks;                            // [n_adapters + 2 most_chunks]: adapter, part, parts (0: no token), place of the adapter's first part among those of several
    float* partial;                          // [2 most_chunks][slices * rank_blocks][16 MT][columns]
};

// Block 0: entries and chunks, and the counters set to zero.  The others: G and H in parts.
constexpr int GP_THREADS = 1024, GP_ROUNDS = 8;
__global__ void __launch_bounds__(GP_THREADS)
adapters_grad_plan_kernel(const Grads p, const float* __restrict__ G, const float* __restrict__ H, uint32_t* __restrict__ g, uint32_t* __restrict__ h, int n_counters) {
    __shared__ int counts[GP_ROUNDS * 32], parts_s[32], several_s[32], total_s;
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x > 0) {
        const long long n = (long long)p.M * p.r, at = (long long)(blockIdx.x - 1) * GP_THREADS + threadIdx.x;
        if (2 * at >= n) return;
        const float2 v[2] = {__ldcg(reinterpret_cast<const float2*>(G) + at), __ldcg(reinterpret_cast<const float2*>(H) + at)};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t* to = k ? h : g;
            float x = v[k].x, y = v[k].y;
#pragma unroll
            for (int i = 0; i < GR_PARTS; ++i) {
                const uint32_t w = bf16x2(x, y);
                to[i * (n / 2) + at] = w;
                x -= bf16_lo(w);                                       // (nothing is left of what is not finite)
                y -= bf16_hi(w);
                x = fabsf(x) < INFINITY ? x : 0.f;
                y = fabsf(y) < INFINITY ? y : 0.f;
            }
        }
        return;
    }
    for (int i = threadIdx.x; i < n_counters; i += GP_THREADS) p.counters[i] = 0u;
    for (int i = threadIdx.x; i < p.n_adapters; i += GP_THREADS) p.counts[i] = 0;
    __threadfence_block();
    __syncthreads();
    int n_entries = 0;
    for (int w0 = 0; w0 < p.M; w0 += GP_ROUNDS * GP_THREADS) {
        int a[GP_ROUNDS];
        uint32_t mask[GP_ROUNDS];
#pragma unroll
        for (int k = 0; k < GP_ROUNDS; ++k) {
            const int t = w0 + k * GP_THREADS + threadIdx.x;
            a[k] = t < p.M ? __ldg(p.adapter_of + t) : -1;
        }
#pragma unroll
        for (int k = 0; k < GP_ROUNDS; ++k) {
            if (a[k] >= p.n_adapters) a[k] = -1;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, a[k]) & (lane < 16 ? 0x0000FFFFu : 0xFFFF0000u);
            mask[k] = a[k] >= 0 && (same & ((1u << lane) - 1u)) == 0 ? same : 0u;      // the first token of an entry
            const int n = __popc(__ballot_sync(0xFFFFFFFFu, mask[k] != 0));
            if (lane == 0) counts[k * 32 + warp] = n;
        }
        __syncthreads();
        if (warp == 0) {                                               // counts -> places
            int mine[GP_ROUNDS], sum = 0;
#pragma unroll
            for (int k = 0; k < GP_ROUNDS; ++k) { mine[k] = sum; sum += counts[lane * GP_ROUNDS + k]; }
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane >= o) before += x;
            }
            if (lane == 31) total_s = before;
#pragma unroll
            for (int k = 0; k < GP_ROUNDS; ++k) counts[lane * GP_ROUNDS + k] = before - sum + mine[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < GP_ROUNDS; ++k) {
            const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mask[k] != 0);
            if (mask[k] != 0) {
                const int t = w0 + k * GP_THREADS + warp * 32 + lane;
                p.entries[n_entries + counts[k * 32 + warp] + __popc(firsts & ((1u << lane) - 1u))] =
                    make_uint2((unsigned)a[k], (uint32_t)(t / 16) << 16 | (lane < 16 ? mask[k] : mask[k] >> 16));
                atomicAdd(p.counts + a[k], 1);
            }
        }
        n_entries += total_s;
        __syncthreads();
    }
    const int tiles = max(GR_MIN_TILES, (n_entries + p.most_chunks - 1) / p.most_chunks);
    int n_chunks = 0, n_several = 0;
    for (int a0 = 0; a0 < p.n_adapters; a0 += GP_THREADS) {
        const int a = a0 + threadIdx.x;
        const int count = a < p.n_adapters ? *(volatile int*)(p.counts + a) : 0;
        const int n = a < p.n_adapters ? max(1, (count + tiles - 1) / tiles) : 0, several = n > 1 ? n : 0;   // (one without tokens has a chunk that writes its zeros)
        int before = n, before_several = several;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, before, o), y = __shfl_up_sync(0xFFFFFFFFu, before_several, o);
            if (lane >= o) { before += x; before_several += y; }
        }
        if (lane == 31) { parts_s[warp] = before; several_s[warp] = before_several; }
        __syncthreads();
        int at = n_chunks + before - n, at_several = n_several + before_several - several;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) { at += parts_s[w]; at_several += several_s[w]; }
            n_chunks += parts_s[w];
            n_several += several_s[w];
        }
        for (int i = 0; i < n; ++i) p.chunks[at + i] = make_int4(a, i, count > 0 ? n : 0, at_several);
        __syncthreads();
    }
    if (threadIdx.x == 0) { p.counters[1] = (unsigned)n_entries; p.counters[2] = (unsigned)tiles; p.counters[3] = (unsigned)n_chunks; }
}

template <int MT>
struct GradTile {
    static constexpr int COLS = MT == 1 ? 128 : 64, RANKS = 16 * MT, PITCH = COLS + 4;    // PITCH: of the sums in shared memory
    static constexpr int V_BYTES = 16 * COLS * 2, P_BYTES = 16 * RANKS * 2, STAGE = V_BYTES + GR_PARTS * P_BYTES;
    static constexpr size_t RING = (size_t)GR_WARPS * GR_STAGES * STAGE, SUMS = sizeof(float) * GR_WARPS * RANKS * PITCH;
    static constexpr size_t SMEM = RING > SUMS ? RING : SUMS;
};

constexpr int GR_LIST = 512, GR_READ = 2;                                  // entries of a chunk that are worked on at a time; entries that a thread reads at a time

template <int MT>
__device__ __forceinline__ void grad_task(const Grads& p, int task, int n_entries, int chunk_tiles, uint8_t* smem, uint32_t* list, int* counts, int* is_last) {
    using Tile = GradTile<MT>;
    constexpr int COLS = Tile::COLS, RANKS = Tile::RANKS, PITCH = Tile::PITCH, CT = COLS / 8;
    float* red = reinterpret_cast<float*>(smem);                       // [warps][RANKS][PITCH], where the rings were
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, row8 = lane & 7, quarter = lane >> 3;
    const int blocks = p.slices * p.rank_blocks, block = task % blocks, slice = block / p.rank_blocks, j0 = block % p.rank_blocks * RANKS;
    const int4 chunk = __ldcg(p.chunks + task / blocks);
    const int adapter = chunk.x, part = chunk.y, parts = chunk.z;
    const bool of_x = slice < p.slices_x;
    const int C = of_x ? p.K : p.N, c0 = (of_x ? slice : slice - p.slices_x) * COLS, M = p.M, r = p.r;
    const bf16 *V = of_x ? p.X : p.dY, *P = of_x ? p.G : p.H;
    const uint32_t ring = smem_u32(smem) + warp * GR_STAGES * Tile::STAGE;
    // what a lane copies: a 16-byte piece of every PER-th row of V, and pieces of all parts of P.  Pieces are XORed by row.
    constexpr int PIECES = COLS / 8, PER = 32 / PIECES, P_PIECES = RANKS / 8;
    const int v_row = lane / PIECES, v_piece = lane % PIECES;
    const bool v_in = c0 + 8 * v_piece < C;
    const int p_row = lane / P_PIECES % 16, p_piece = lane % P_PIECES;
    const bool p_in = j0 + 8 * p_piece < r;
    if (parts == 0) {                                                  // an adapter without tokens
        if (p.accumulate) return;
        for (int quad = threadIdx.x; quad < RANKS * COLS / 4; quad += 32 * GR_WARPS) {
            const int j = of_x ? quad / (COLS / 4) : 4 * (quad % (RANKS / 4)), c = of_x ? 4 * (quad % (COLS / 4)) : quad / (RANKS / 4);
            if (j0 + j < r && c0 + c < C)
                *reinterpret_cast<float4*>(of_x ? p.dA + ((size_t)adapter * r + j0 + j) * p.K + c0 + c : p.dB + ((size_t)adapter * p.N + c0 + c) * r + j0 + j) =
                    make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    const int lo = part * chunk_tiles, hi = lo + chunk_tiles;          // of the adapter's entries
    float acc[MT][CT][4];
    auto pass = [&](auto again) {                                      // whether a sum is not finite
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < CT; ++t) acc[mt][t][0] = acc[mt][t][1] = acc[mt][t][2] = acc[mt][t][3] = 0.f;
        int seen = 0;                                                  // of the adapter's entries
        for (int e0 = 0; e0 < n_entries && seen < hi;) {
            // the chunk's entries from e0 on, until the list is full
            int total = 0;
            for (; e0 < n_entries && seen < hi && total <= GR_LIST - GR_READ * 32 * GR_WARPS;) {
                uint2 e[GR_READ];
                uint32_t votes[GR_READ];
#pragma unroll
                for (int k = 0; k < GR_READ; ++k) {
                    const int i = e0 + (k * GR_WARPS + warp) * 32 + lane;
                    e[k] = i < n_entries ? __ldcg(p.entries + i) : make_uint2(0xFFFFFFFFu, 0u);
                }
#pragma unroll
                for (int k = 0; k < GR_READ; ++k) {
                    votes[k] = __ballot_sync(0xFFFFFFFFu, e[k].x == (unsigned)adapter);
                    if (lane == 0) counts[k * GR_WARPS + warp] = __popc(votes[k]);
                }
                __syncthreads();
                int all = 0;
#pragma unroll
                for (int k = 0; k < GR_READ; ++k)
#pragma unroll
                    for (int w = 0; w < GR_WARPS; ++w) {
                        const int ordinal = seen + all + __popc(votes[k] & ((1u << lane) - 1u));
                        if (w == warp && ((votes[k] >> lane) & 1u) && ordinal >= lo && ordinal < hi) list[total + ordinal - max(lo, seen)] = e[k].y;
                        all += counts[k * GR_WARPS + w];
                    }
                total += max(0, min(hi, seen + all) - max(lo, seen));
                seen += all;
                e0 += GR_READ * GR_WARPS * 32;
                __syncthreads();
            }
            const int mine = warp < total ? (total - warp + GR_WARPS - 1) / GR_WARPS : 0;
            uint32_t to = ring, from = ring;                           // the stages that are filled and read next
            auto after = [&](uint32_t stage) { return stage + Tile::STAGE == ring + GR_STAGES * Tile::STAGE ? ring : stage + Tile::STAGE; };
            auto load = [&](int i) {
                const uint32_t entry = list[warp + i * GR_WARPS];
                const int t0 = (int)(entry >> 16) * 16;
                const bf16* v = V + (size_t)(t0 + v_row) * C + (v_in ? c0 + 8 * v_piece : 0);
#pragma unroll
                for (int n = 0; n < 16 / PER; ++n) {
                    const int row = n * PER + v_row;
                    const bool in = v_in && ((entry >> row) & 1u);
                    copy16(to + row * (COLS * 2) + ((v_piece ^ (row & 7)) << 4), in ? v : V, in);      // (128 or 256 bytes to a row)
                    v += (size_t)PER * C;
                }
                const bf16* low = P + (size_t)(t0 + p_row) * r + (p_in ? j0 + 8 * p_piece : 0);
                const bool in = p_in && ((entry >> p_row) & 1u);
                const uint32_t p_to = to + Tile::V_BYTES + p_row * (RANKS * 2) + ((p_piece ^ (p_row * P_PIECES / 8 % P_PIECES)) << 4);
                // (a part is 32 pieces, or 64: then eight rows further on as well, with the same XOR)
                const bool in8 = p_in && ((entry >> ((p_row + 8) & 31)) & 1u);
#pragma unroll
                for (int k = 0; k < GR_PARTS; ++k) {
                    copy16(p_to + k * Tile::P_BYTES, in ? low + (size_t)k * M * r : P, in);
                    if constexpr (P_PIECES == 4) copy16(p_to + k * Tile::P_BYTES + 8 * (RANKS * 2), in8 ? low + ((size_t)k * M + 8) * r : P, in8);
                }
                to = after(to);
            };
#pragma unroll
            for (int i = 0; i < GR_STAGES - 1; ++i) {
                if (i < mine) load(i);
                copy_commit();
            }
            const uint32_t v_off = (row8 + 8 * (quarter & 1)) * (COLS * 2), v_xor = (uint32_t)((quarter >> 1) ^ row8) << 4;
            const int a_row = row8 + 8 * (quarter >> 1);
#pragma unroll 1
            for (int i = 0; i < mine; ++i) {
                copy_wait<GR_STAGES - 2>();
                __syncwarp();                                          // tile i is there, tile i - 1 has been read by every lane
                if (i + GR_STAGES - 1 < mine) load(i + GR_STAGES - 1);
                copy_commit();
                const uint32_t v = from, pp = v + Tile::V_BYTES;
                from = after(from);
                uint32_t a[GR_PARTS][MT][4];
#pragma unroll
                for (int half = 0; half < GR_PARTS; ++half)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {                  // ranks 0 - 7, 8 - 15 of tokens 0 - 7; then of 8 - 15
                        const int piece = 2 * mt + (quarter & 1);
                        ldmatrix4<true>(pp + half * Tile::P_BYTES + a_row * (RANKS * 2) + ((piece ^ (a_row * P_PIECES / 8 % P_PIECES)) << 4), a[half][mt][0],
                                        a[half][mt][1], a[half][mt][2], a[half][mt][3]);
                    }
                uint32_t b[CT / 2][4];                                 // tokens 0 - 7, 8 - 15 of columns 16 t ..; then of the next eight
#pragma unroll
                for (int t = 0; t < CT / 2; ++t) ldmatrix4<true>(v + v_off + (v_xor ^ (t << 5)), b[t][0], b[t][1], b[t][2], b[t][3]);
#pragma unroll
                for (int k = 0; k < GR_PARTS; ++k) {                   // (part by part: a sum's products are far apart)
                    if constexpr (decltype(again)::value)
                        if (k == 1)
#pragma unroll
                            for (int t = 0; t < CT / 2; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) b[t][i] = finite_pair(b[t][i]);
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
                            mma_bf16_16816(acc[mt][t], a[k][mt][0], a[k][mt][1], a[k][mt][2], a[k][mt][3], b[t / 2][2 * (t % 2)], b[t / 2][2 * (t % 2) + 1]);
                }
            }
            copy_wait<0>();
            __syncthreads();                                           // the list is written again, the sums where the rings are
        }
        float worst = 0.f;                                             // (x - x is 0, or a NaN)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) worst += acc[mt][t][k] - acc[mt][t][k];
        return __syncthreads_or(worst != 0.f) != 0;
    };
    if (pass(std::false_type{})) pass(std::true_type{});
    // [mt][t][c]: rank 16 mt + g (+ 8 where c >= 2), column 8 t + 2 q + c % 2
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2*>(red + ((size_t)warp * RANKS + 16 * mt + 8 * h + g) * PITCH + 8 * t + 2 * q) =
                    make_float2(acc[mt][t][2 * h], acc[mt][t][2 * h + 1]);
    __syncthreads();
    // From here on four values at a time, in the order of the output: A's gradient along the columns, B's along the ranks.
    constexpr int QUADS = RANKS * COLS / 4;
    auto place = [&](int quad, int& j, int& c) {
        if (of_x) { j = quad / (COLS / 4); c = 4 * (quad % (COLS / 4)); }
        else { c = quad / (RANKS / 4); j = 4 * (quad % (RANKS / 4)); }
    };
    auto sum = [&](int quad) {
        int j, c;
        place(quad, j, c);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < GR_WARPS; ++w) {
            const float* from = red + (w * RANKS + j) * PITCH + c;
            if (of_x) {
                const float4 x = *reinterpret_cast<const float4*>(from);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            } else {
                v.x += from[0]; v.y += from[PITCH]; v.z += from[2 * PITCH]; v.w += from[3 * PITCH];
            }
        }
        return v;
    };
    const bool split = parts > 1;
    const size_t apart = (size_t)blocks * QUADS;                       // from one chunk's sums to the next one's
    float4* partial = reinterpret_cast<float4*>(p.partial) + (size_t)chunk.w * apart + (size_t)block * QUADS;
    if (split) {
        for (int quad = threadIdx.x; quad < QUADS; quad += 32 * GR_WARPS) __stcg(partial + part * apart + quad, sum(quad));
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            *is_last = atomicAdd(p.counters + 4 + (size_t)chunk.w * blocks + block, 1u) == (unsigned)parts - 1u;
            __threadfence();
        }
        __syncthreads();
        if (!*is_last) return;
    }
    const float s = p.scales[adapter];
    constexpr int EACH = QUADS / (32 * GR_WARPS);
    float4 v[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int quad = threadIdx.x + i * 32 * GR_WARPS;
        v[i] = split ? __ldcg(partial + quad) : sum(quad);
    }
    if (split)
#pragma unroll 4
        for (int k = 1; k < parts; ++k)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const float4 x = __ldcg(partial + k * apart + threadIdx.x + i * 32 * GR_WARPS);
                v[i].x += x.x; v[i].y += x.y; v[i].z += x.z; v[i].w += x.w;
            }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        int j, c;
        place(threadIdx.x + i * 32 * GR_WARPS, j, c);
        if (j0 + j >= r || c0 + c >= C) continue;                      // (four are inside or outside together)
        float4* dst = reinterpret_cast<float4*>(of_x ? p.dA + ((size_t)adapter * r + j0 + j) * p.K + c0 + c : p.dB + ((size_t)adapter * p.N + c0 + c) * r + j0 + j);
        float4 x = make_float4(s * v[i].x, s * v[i].y, s * v[i].z, s * v[i].w);
        if (p.accumulate) {
            const float4 old = *dst;
            x.x += old.x; x.y += old.y; x.z += old.z; x.w += old.w;
        }
        *dst = x;
    }
}

template <int MT>
__global__ void __launch_bounds__(32 * GR_WARPS, GR_BLOCKS)
adapters_grad_kernel(const Grads p) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint32_t list[GR_LIST];
    __shared__ int counts[GR_READ * GR_WARPS], claimed, is_last;
    pdl_launch_dependents();
    pdl_wait();
    const int n_entries = (int)__ldcg(p.counters + 1), chunk_tiles = (int)__ldcg(p.counters + 2);
    const int n_tasks = p.slices * p.rank_blocks * (int)__ldcg(p.counters + 3);
    // the first task is the block's own number; the next is claimed while one is worked on
    for (int task = blockIdx.x; task < n_tasks;) {
        if (threadIdx.x == 0) claimed = (int)(gridDim.x + atomicAdd(p.counters, 1u));
        grad_task<MT>(p, task, n_entries, chunk_tiles, smem, list, counts, &is_last);
        __syncthreads();
        task = claimed;
        __syncthreads();                                               // shared memory is written again
    }
}

template <bool L_IS_A, int NT, int NB, int CTAS>
int down_impl(const Products& p, cudaStream_t st) {
    constexpr size_t smem = DownTile<L_IS_A, NT, NB, CTAS>::SMEM;
    static SmemLimit limit;
    auto kern = adapters_down_kernel<L_IS_A, NT, NB, CTAS>;
    if (!limit.raise(kern, smem)) return QLORA_ERR_CUDA;
    // helpers come last: on what the tiles leave free, or when the first of them are through
    const int tiles = (p.M + 16 * NB - 1) / (16 * NB) * CTAS, room = (NT <= 4 ? 2 : 1) * sm_count() - tiles;
    const int helpers = (room < DN_HELPERS ? DN_HELPERS : room > sm_count() ? sm_count() : room) / CTAS * CTAS;
    if (launch_pdl(adapters_groups_kernel, dim3(1), dim3(SORT_THREADS), 0, st, 1, p.M, p.n_adapters, p.adapter_of, p.groups) != cudaSuccess) return QLORA_ERR_CUDA;
    return launch_pdl(kern, dim3(tiles + helpers), dim3(32 * DN_WARPS), smem, st, CTAS, p, tiles) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

template <bool FROM_B, int KS, int UB>
int up_impl(const Products& p, cudaStream_t st) {
    const int columns = (p.C + 32 * UB * UP_WARPS - 1) / (32 * UB * UP_WARPS), tiles = (p.M + UP_ROWS - 1) / UP_ROWS;
    // Tiles to a block: up_blocks(KS) run on an SM, so it is waves of blocks times the tiles of one, and about two tiles' time for a block to begin.
    const long long room = up_blocks(KS) * sm_count();
    int each = 1;
    for (long long i = 1, best = 1ll << 60; i <= 64; ++i) {
        const long long blocks = (tiles + i - 1) / i * columns, cost = (blocks + room - 1) / room * (i + 2);
        if (cost < best) { best = cost; each = (int)i; }
    }
    return launch_pdl(adapters_up_kernel<FROM_B, KS, UB>, dim3((tiles + each - 1) / each, columns), dim3(32 * UP_WARPS), 0, st, 1, p, each) == cudaSuccess
               ? QLORA_OK : QLORA_ERR_CUDA;
}

template <bool FORWARD, int NT, int ROWS, int CTAS>
int few_impl(const Products& p, cudaStream_t st) {
    return launch_pdl(adapters_few_kernel<FORWARD, NT, ROWS, CTAS>, dim3((p.M + ROWS - 1) / ROWS * CTAS), dim3(32 * FEW_WARPS), 0, st, 1, p) == cudaSuccess
               ? QLORA_OK : QLORA_ERR_CUDA;   // (the cluster's width is an attribute of the kernel)
}

template <bool FORWARD, int NT, int NB, int KS, int UB>
int products(const Products& p, cudaStream_t st) {
    // A cluster for every token, as wide as lets all of them run at a time (two blocks to an SM).  Then, up to rank 16, for every four tokens: 256 tokens of 4 prompts
    // take 14 us both ways, those of 32 adapters in turn 30 us instead of 25, and of 256 adapters 35 instead of 67; at rank 64 it is 40 instead of 15, 109
    // instead of 30 and 146 instead of 124 (4096 x 4096).
    const int room = 2 * sm_count();
    if (p.Out != nullptr && (2 * p.M <= room || (NT <= 2 && p.M <= FEW_TOKENS))) {
        if (8 * p.M <= room) return few_impl<FORWARD, NT, 1, 8>(p, st);
        if (4 * p.M <= room) return few_impl<FORWARD, NT, 1, 4>(p, st);
        if (2 * p.M <= room) return few_impl<FORWARD, NT, 1, 2>(p, st);
        if constexpr (NT <= 2) return few_impl<FORWARD, NT, 4, 4>(p, st);
    }
    // blocks to a tile: while all of them run at a time
    const int tiles = (p.M + 16 * NB - 1) / (16 * NB), at_a_time = (NT <= 4 ? 2 : 1) * sm_count();
    const int rc = 4 * tiles <= at_a_time ? down_impl<FORWARD, NT, NB, 4>(p, st) : 2 * tiles <= at_a_time ? down_impl<FORWARD, NT, NB, 2>(p, st) : down_impl<FORWARD, NT, NB, 1>(p, st);
    return rc != QLORA_OK || p.Out == nullptr ? rc : up_impl<FORWARD, KS, UB>(p, st);
}

// Slices and chunks of the gradients: as many chunks as give every SM all its blocks twice, two at least.  (A task's own cost is that of a dozen tiles: with sixteen chunks at
// least, 8192 tokens at rank 64, 4096 x 11008, took 220 us instead of 165, 22 prompts 124 instead of 96; with tasks for four or eight turns of blocks 159 and 181, 107 and 124.)
void cut_grads(Grads& p) {
    const int columns = p.r <= 16 ? GradTile<1>::COLS : GradTile<2>::COLS, ranks = p.r <= 16 ? GradTile<1>::RANKS : GradTile<2>::RANKS;
    p.slices_x = (p.K + columns - 1) / columns;
    p.slices = p.slices_x + (p.N + columns - 1) / columns;
    p.rank_blocks = (p.r + ranks - 1) / ranks;
    const int blocks = p.slices * p.rank_blocks, wanted = 2 * GR_BLOCKS * sm_count();
    p.most_chunks = blocks == 0 ? 2 : (wanted + blocks - 1) / blocks;
    p.most_chunks = p.most_chunks < 2 ? 2 : p.most_chunks > 128 ? 128 : p.most_chunks;
}

struct GradScratch { size_t g, h, counters, entries, counts, chunks, partial, total; };
GradScratch grad_scratch(const Grads& p) {
    const size_t blocks = (size_t)p.slices * p.rank_blocks, several = 2 * (size_t)p.most_chunks;
    const size_t tile = p.r <= 16 ? GradTile<1>::RANKS * GradTile<1>::COLS : GradTile<2>::RANKS * GradTile<2>::COLS;
    GradScratch s;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    s.g = take((size_t)GR_PARTS * p.M * p.r * 2);
    s.h = take((size_t)GR_PARTS * p.M * p.r * 2);
    s.counters = take(4 * (4 + several * blocks));
    s.entries = take((size_t)p.M * sizeof(uint2));
    s.counts = take((size_t)p.n_adapters * 4);
    s.chunks = take(((size_t)p.n_adapters + several) * sizeof(int4));
    s.partial = take(several * blocks * tile * sizeof(float));
    s.total = at;
    return s;
}

template <int MT>
int grad_impl(const Grads& p, cudaStream_t st) {
    static SmemLimit limit;
    auto kern = adapters_grad_kernel<MT>;
    if (!limit.raise(kern, GradTile<MT>::SMEM)) return QLORA_ERR_CUDA;
    return launch_pdl(kern, dim3(GR_BLOCKS * sm_count()), dim3(32 * GR_WARPS), GradTile<MT>::SMEM, st, 1, p) == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

}  // namespace

size_t adapters_scratch_bytes(int M, int r) { return (size_t)M * split_pairs(r) * sizeof(uint2) + 8 + (size_t)M * (sizeof(int2) + sizeof(int)); }

int launch_adapters(bool forward, int M, int T, int C, int r, int n_adapters, const void* In, const int32_t* adapter_of, const void* L1, const void* L2,
                    const float* scales, const void* Base, void* Out, float* P, void* scratch, cudaStream_t st) {
    char* groups = static_cast<char*>(scratch) + (size_t)M * split_pairs(r) * sizeof(uint2);
    const Products p{M, T, C, r, n_adapters, (const bf16*)In, adapter_of, (const bf16*)L1, (const bf16*)L2, scales, (const bf16*)Base, (bf16*)Out, P,
                     Out != nullptr ? (uint2*)scratch : nullptr, Groups{(int*)groups, (int2*)(groups + 8), (int*)(groups + 8 + (size_t)M * sizeof(int2))}};
#define QLORA_PRODUCTS(NT, NB, KS, UB) return forward ? products<true, NT, NB, KS, UB>(p, st) : products<false, NT, NB, KS, UB>(p, st)
    if (r <= 8) QLORA_PRODUCTS(1, 1, 1, 2);
    if (r <= 16) QLORA_PRODUCTS(2, 1, 1, 2);
    if (r <= 32) QLORA_PRODUCTS(4, 1, 2, 2);
    QLORA_PRODUCTS(8, 2, 4, 2);
#undef QLORA_PRODUCTS
}

size_t adapters_grad_scratch_bytes(int M, int K, int N, int r, int n_adapters) {
    Grads p{};
    p.M = M; p.K = K; p.N = N; p.r = r; p.n_adapters = n_adapters;
    cut_grads(p);
    return grad_scratch(p).total;
}

int launch_adapters_grads(int M, int K, int N, int r, int n_adapters, const void* X, const void* dY, const int32_t* adapter_of, const float* scales,
                          const float* H, const float* G, float* dA, float* dB, int accumulate, void* scratch, cudaStream_t st) {
    Grads p{};
    p.M = M; p.K = K; p.N = N; p.r = r; p.n_adapters = n_adapters;
    p.X = (const bf16*)X; p.dY = (const bf16*)dY; p.adapter_of = adapter_of; p.scales = scales; p.dA = dA; p.dB = dB; p.accumulate = accumulate;
    cut_grads(p);
    const GradScratch s = grad_scratch(p);
    char* at = static_cast<char*>(scratch);
    p.G = reinterpret_cast<bf16*>(at + s.g);
    p.H = reinterpret_cast<bf16*>(at + s.h);
    p.counters = reinterpret_cast<unsigned*>(at + s.counters);
    p.entries = reinterpret_cast<uint2*>(at + s.entries);
    p.counts = reinterpret_cast<int*>(at + s.counts);
    p.chunks = reinterpret_cast<int4*>(at + s.chunks);
    p.partial = reinterpret_cast<float*>(at + s.partial);
    const long long pairs = (long long)M * r / 2;
    if (launch_pdl(adapters_grad_plan_kernel, dim3((unsigned)(1 + (pairs + GP_THREADS - 1) / GP_THREADS)), dim3(GP_THREADS), 0, st, 1, p, G, H,
                   reinterpret_cast<uint32_t*>(at + s.g), reinterpret_cast<uint32_t*>(at + s.h), (int)((s.entries - s.counters) / 4)) != cudaSuccess)
        return QLORA_ERR_CUDA;
    return r <= 16 ? grad_impl<1>(p, st) : grad_impl<2>(p, st);
}

}  // namespace qlora
