// Cross entropy of the model's head from the hidden states, and its gradient with respect to them, without the logits in memory.
//   z = h W^T,   loss = log sum_v exp z_v - z_label,   dh = d_loss (sum_v p_v W_v - W_label),   p = softmax(z)
//
// Two products, 2 T V D operations each, and nothing is computed twice: the probabilities of a piece of the vocabulary (4096 entries) go to the second
// product as P = exp(z - ref), bf16, through a small ring that stays in L2, with one reference per token for the whole vocabulary, which is known
// before the row's true maximum is: the largest of its first 256 logits (the label's apart) and 40 ln 2 more.  The sums over the pieces then need no rescaling -- they are
// divided by the row's sum of P at the end -- and bf16 has the range of fp32: nothing is lost while the row's maximum lies up to 120 ln 2 = 83 above
// those first logits, and what flushes to zero is below 2^-86 of the largest.  A token whose largest logit lies further above is found at the end, and its
// block of 256 tokens is computed again from its true maximum (by a second launch of the same kernel, which ends at once where there is none).
//
// The label's own term is kept out of P: p_label - 1 = -(sum of the others) / sum has no cancellation, and where a token is almost
// certain the gradient would otherwise be the rounding error of P.  And the others' rows are weighed with sum P / sum of the rounded P, so that the weights of all
// rows add up to nothing: a vector that all rows of the head share would otherwise come out times the rounding error (20 standard deviations of the rows'
// own parts, logits that spread by 4: 5e-2 of a token's gradient, now 2e-3, which is the result's own rounding).
//
// Rounding: P to bf16 (a relative error of 2^-9 on average over many terms of either sign), dh to bf16; everything else is fp32.
//
// One persistent kernel: a pair of CTAs (two SMs) claims items of both products from one counter (head_plan.h), so there is no wave to wait for
// between the products or the pieces.  An item is a tile of 256 x 256 (tcgen05.mma.cta_group::2, M = 256, N = 256; 128 rows and half of the other
// operand per CTA), operands staged by TMA in six stages (more for few rows) of 64 contraction elements, accumulators in tensor memory twice, so that the
// epilogue of an item runs beside the products of the next.  What an item needs from others (probabilities of its rows, the previous piece's sums, a free slot
// of the ring, the reference) it waits for through counters in the workspace; those items were claimed earlier, so the wait ends
// whichever CTAs share the GPU.  Every wait is bounded.
//
// Bound by the tensor cores.  2048 tokens, 32000 entries, 4096 features, a launch by itself: the loss 336 - 338 us (1590 TFLOP/s, the pipe 87 % active), with the gradient
// 698 - 727 us (1477 - 1539), of which writing the probabilities is some 30 and adding to the sums 5; calls in a loop, under the power limit, 409 - 422 and 896 - 940 us in all,
// by the GPU.  Pieces of 2048 and 8192 entries: 761 and 750 us where these take 698; four stages 738.  The kernel that finishes takes 23 - 25 us beside that, the second
// launches 7.  Few tokens are bound by reading the head in whole tiles: 16 tokens 60 us for 262 MB (4.4 TB/s), 125 tiles in two rounds of 74 pairs, the second with
// 51 of them reading, and 11 us of launches, preparing and finishing.  Blocks of rows are whole: 520 tokens are 2.03 of them and cost 3.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"
#include "device_state.h"
#include "f32x2.cuh"
#include "head_plan.h"
#include "launch.h"
#include "tcgen05.cuh"

namespace qlora {

__device__ unsigned int g_head_status = 0;   // sticky; bit 0: a wait gave up

namespace {

typedef __nv_bfloat16 bf16;

constexpr int HL_THREADS = 256, HL_MAX_STAGES = 12, HL_EPI_WARP0 = 4, HL_EPI_WARPS = 4, HL_CLAIMS = 4;
constexpr uint32_t HL_HALF = 128 * 64 * 2;                            // one CTA's part of an operand
constexpr uint32_t HL_SLICE = 4096;                                   // staging of an epilogue warp
constexpr uint32_t HL_RING = 6 * 2 * HL_HALF, HL_OFF_SLICES = HL_RING, HL_OFF_BARS = HL_OFF_SLICES + HL_EPI_WARPS * HL_SLICE;
constexpr size_t HL_SMEM = HL_OFF_BARS + 512 + 1024;
constexpr int HL_WAIT_US = 250000;
constexpr uint32_t HL_SPINS = 1u << 26;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f, MOST = 3.402823466e38f;
// The tensor cores cut their fp32 sums off towards zero at every step, which is an expected loss, not a random one: logits of random terms came out smaller by
// 1.0e-9 of their size per contraction element (measured against 64-bit sums at 1024, within 12 %, and from 4096 to 262144, within 2 %;
// below it drowns in fp32's own rounding).  The exponentials' scale takes the expected part back: mean error of a logit at 4096 elements 4e-6 -> 2e-9, at 16384 1.6e-5 -> 1.2e-7;
// of the losses at 4096, root of the mean square, 2.2e-6 -> 8e-7.
// It is the wrong thing for other sums: exact ones (few features that are not zero, whole numbers) lose nothing and come out larger by it, and those whose terms
// have one sign lose more (in all 3e-9 per element at 4096, 4.5e-9 at 16384).  So it grows with the length up to 16384 only, 1.6e-5 of a logit.
constexpr float CUT_OFF = 1.0e-9f;
constexpr int CUT_OFF_LENGTH = 16384;
constexpr float REF_ABOVE = 40.f * LN2;      // the reference over the largest of the first logits
constexpr float REF_REACH = 80.f * LN2;      // how far a logit may lie above it: sums of 2^24 terms times weights below 2^20 stay finite

struct HeadParams {
    HeadPlan plan;
    int again;                               // the second launch: only blocks that are to be done again
    int tokens, copies;                      // copies: the hidden states are copied even where every token has a label
    int wait_limit_us;
    // A stage: the rows' operand (row_bytes) and the head's.  Up to 128 tokens it has room for those rows alone, so that more stages are under way, which is what
    // reading the head takes: the products read on into whatever lies behind, for rows of the result that nobody takes.
    uint32_t stages, stage, row_bytes;
    float scale;                             // log2 e, and what the products' sums lose (CUT_OFF)
    size_t padded;                           // rows of the buffers
    unsigned* counters;
    const int* label;
    float *ref, *label_logit;
    float2* tile_stats;                      // [rows][tiles]: the largest logit, the sum
    float* tile_rounded;                     // [rows][tiles], with the gradient: the sum of what enters its product
    bf16* probs;
    float* sums;
};

// Where the counters lie.
__device__ __forceinline__ unsigned* ref_known(const HeadParams& p) { return p.counters + 4; }
__device__ __forceinline__ unsigned* to_do_again(const HeadParams& p) { return p.counters + 4 + p.plan.blocks_max; }
__device__ __forceinline__ unsigned* logits_done(const HeadParams& p) {
    const size_t set = (size_t)head_div_up(p.plan.blocks_max, kHeadChunk) * p.plan.pieces * kHeadChunk;
    return p.counters + 4 + 2 * p.plan.blocks_max + (p.again ? 2 * set : 0);
}
__device__ __forceinline__ unsigned* grads_done(const HeadParams& p) {
    return logits_done(p) + (size_t)head_div_up(p.plan.blocks_max, kHeadChunk) * p.plan.pieces * kHeadChunk;
}

__device__ __forceinline__ bool gave_up(volatile int* abort_flag) {
    *abort_flag = 1;
    atomicOr(&g_head_status, 1u);
    return false;
}
// Waits of a whole warp: on a barrier (all lanes see the completed phase), and on a counter in global memory (lane 0 reads, the warp's
// barrier hands it on).  They give up after abort_flag[1] microseconds.
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    uint64_t t0 = 0;
    for (uint32_t i = 0; i < HL_SPINS; ++i) {
        if (__all_sync(0xFFFFFFFFu, mbar_try_wait_cluster(bar, parity) != 0u)) return true;
        if ((i & 63u) == 63u) {
            if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) return false;
            const uint64_t now = __shfl_sync(0xFFFFFFFFu, global_ns(), 0);
            if (t0 == 0) t0 = now;
            else if (now - t0 > (uint64_t)abort_flag[1] * 1000ull) break;
        }
    }
    return gave_up(abort_flag);
}
__device__ __forceinline__ bool poll_counter(const unsigned* counter, unsigned target, volatile int* abort_flag) {
    uint64_t t0 = 0;
    const int lane = threadIdx.x & 31;
    for (uint32_t i = 0; i < HL_SPINS; ++i) {
        unsigned v = 0;
        if (lane == 0) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
        if (__shfl_sync(0xFFFFFFFFu, v, 0) >= target) { __syncwarp(); return true; }
        __nanosleep(100);
        if ((i & 63u) == 63u) {
            if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) return false;
            const uint64_t now = __shfl_sync(0xFFFFFFFFu, global_ns(), 0);
            if (t0 == 0) t0 = now;
            else if (now - t0 > (uint64_t)abort_flag[1] * 1000ull) break;
        }
    }
    return gave_up(abort_flag);
}
__device__ __forceinline__ void arrive_release_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
// An epilogue warp's writes to global memory, counted in where other SMs read them (also through TMA).  Every warp counts for itself, so that none
// waits for one that has given up: a tile is COUNTS_PER_TILE.
constexpr unsigned COUNTS_PER_TILE = 2 * HL_EPI_WARPS;
__device__ __forceinline__ void publish(unsigned* counter) {
    fence_proxy_async_all();
    __threadfence();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
}

template <bool GRAD>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(HL_THREADS, 1)
head_loss_kernel(const __grid_constant__ CUtensorMap tm_hidden, const __grid_constant__ CUtensorMap tm_rows, const __grid_constant__ CUtensorMap tm_head,
                 const __grid_constant__ CUtensorMap tm_head_t, const __grid_constant__ CUtensorMap tm_probs, const HeadParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag_s[2];
    __shared__ int4 claimed_s[HL_CLAIMS][2];                           // kind (-1 at the end), q, piece, block in its chunk; block, tile, steps
    volatile int* abort_flag = abort_flag_s;
    pdl_launch_dependents();
    if (p.again) {
        pdl_wait();
        if (__ldcg(p.counters + 3) == 0u) return;                      // nothing to do again (the same for both CTAs of a pair)
    }
    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem0 - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t cta = cluster_ctarank();                            // 0 = leader: issues the products, claims the items

    const uint32_t bar_full = smem0 + HL_OFF_BARS;                     // [stages] leader's: both CTAs' operands landed
    const uint32_t bar_empty = bar_full + 8 * HL_MAX_STAGES;           // [stages] both: read by the products (multicast commit)
    const uint32_t bar_acc_full = bar_empty + 8 * HL_MAX_STAGES;           // [2] both: accumulators complete (multicast commit)
    const uint32_t bar_acc_empty = bar_acc_full + 16;                  // [2] leader's: drained by both epilogues
    const uint32_t bar_claim_full = bar_acc_empty + 16;                // [claims] both: an item's number is there
    const uint32_t bar_claim_empty = bar_claim_full + 8 * HL_CLAIMS;   // [claims] leader's: read by every role of both CTAs

    if (threadIdx.x == 0) {
        abort_flag_s[0] = 0;
        abort_flag_s[1] = p.wait_limit_us;
        for (uint32_t i = 0; i < p.stages; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bar_acc_full + 8 * i, 1); mbar_init(bar_acc_empty + 8 * i, 2 * HL_EPI_WARPS); }
        for (int i = 0; i < HL_CLAIMS; ++i) { mbar_init(bar_claim_full + 8 * i, 1); mbar_init(bar_claim_empty + 8 * i, 2 + 1 + 2 * HL_EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                                // the peer's barriers are initialised before anything arrives on them
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;
    pdl_wait();

    const HeadPlan& plan = p.plan;
    const int n_rows = (int)__ldcg(p.counters);
    const HeadRows rows = head_rows(plan, n_rows);
    const int steps_d = head_div_up(plan.D, kHeadStep);
    const uint32_t leader_claim_empty = map_to_cta(bar_claim_empty, 0);
    auto active = [&](int block) { return block < rows.blocks && (!p.again || __ldcg(to_do_again(p) + block) != 0u); };
    auto steps_of = [&](const HeadItem& it) { return it.of_grad ? head_div_up(head_piece_entries(plan, it.piece), kHeadStep) : steps_d; };

    // What every role does for its next item, which the leader has claimed, looked up and waited for: decoding a number costs some hundred cycles of
    // divisions, in which a role that issues copies or products would fall behind.
    struct Item : HeadItem { int steps; };
    Ring claim;
    auto next = [&](Item* it) -> bool {
        if (!poll(bar_claim_full + 8 * claim.slot, claim.phase, abort_flag)) return false;
        const int4 a = claimed_s[claim.slot][0], b = claimed_s[claim.slot][1];
        __syncwarp();
        if (lane == 0) arrive_release_cluster(leader_claim_empty + 8 * claim.slot);
        claim.advance(HL_CLAIMS);
        it->of_grad = a.x; it->q = a.y; it->piece = a.z; it->block_in_chunk = a.w;
        it->block = b.x; it->tile = b.y; it->steps = b.z;
        return a.x >= 0;
    };

    if (warp == 2) {
        // ------------------------------------------------------------------ claims items for the pair
        if (cta == 0) {
            unsigned* counter = p.counters + (p.again ? 2 : 1);
            const uint32_t mine = smem_u32(claimed_s), peer = map_to_cta(mine, 1), peer_full = map_to_cta(bar_claim_full, 1);
            for (bool more = true; more;) {
                if (!poll(bar_claim_empty + 8 * claim.slot, claim.phase ^ 1u, abort_flag)) break;
                int index = -1;
                if (lane == 0) {
                    for (;;) {
                        const unsigned i = atomicAdd(counter, 1u);
                        if ((long long)i >= rows.total) break;
                        const HeadItem it = head_item(plan, rows, i);
                        if (!active(it.block)) continue;               // (the last chunk is shorter, and so is the last piece)
                        if (!it.of_grad && it.tile * plan.tile >= head_piece_entries(plan, it.piece)) continue;
                        index = (int)i;
                        break;
                    }
                }
                index = __shfl_sync(0xFFFFFFFFu, index, 0);
                more = index >= 0;
                HeadItem it{};
                it.of_grad = -1;
                if (more) it = head_item(plan, rows, index);
                if (GRAD && it.of_grad > 0) {                          // its probabilities
                    const unsigned tiles = (unsigned)head_div_up(head_piece_entries(plan, it.piece), plan.tile);
                    if (!poll_counter(logits_done(p) + (size_t)it.q * kHeadChunk + it.block_in_chunk, COUNTS_PER_TILE * tiles, abort_flag)) break;
                }
                if (lane == 0) {
                    const int steps = more ? steps_of(it) : 0;
                    claimed_s[claim.slot][0] = make_int4(it.of_grad, it.q, it.piece, it.block_in_chunk);
                    claimed_s[claim.slot][1] = make_int4(it.block, it.tile, steps, 0);
                    st_cluster_16(peer + 32 * claim.slot, (uint32_t)it.of_grad, (uint32_t)it.q, (uint32_t)it.piece, (uint32_t)it.block_in_chunk);
                    st_cluster_16(peer + 32 * claim.slot + 16, (uint32_t)it.block, (uint32_t)it.tile, (uint32_t)steps, 0u);
                    mbar_arrive(bar_claim_full + 8 * claim.slot);
                    arrive_release_cluster(peer_full + 8 * claim.slot);
                }
                __syncwarp();
                claim.advance(HL_CLAIMS);
            }
        }
    } else if (warp == 0) {
        // ------------------------------------------------------------------ TMA: both operands of this CTA
        Ring ring;
        const uint32_t leader_full = map_to_cta(bar_full, 0);
        const CUtensorMap* of_rows = n_rows == p.tokens && !p.copies ? &tm_hidden : &tm_rows;
        Item it;
        while (next(&it)) {
            const int steps = it.steps;
            if (GRAD && it.of_grad) fence_proxy_async_all();           // (what it reads was written by other SMs' ordinary stores)
            const int row0 = it.of_grad ? ((it.q % plan.ring) * plan.chunk_max + it.block_in_chunk) * kHeadTile + (int)cta * 128 : it.block * kHeadTile + (int)cta * 128;
            const int other0 = it.of_grad ? it.tile * kHeadTile + (int)cta * 128 : it.piece * plan.piece + it.tile * plan.tile + (int)cta * (plan.tile / 2);
            // (a CTA none of whose rows are there leaves its part of the operand as it is: its rows of the result are not used)
            const bool here = it.block * kHeadTile + (int)cta * 128 < n_rows, there = it.block * kHeadTile + 128 < n_rows;
            const uint32_t bytes = (there ? 2 : 1) * p.row_bytes + (it.of_grad ? 2 * HL_HALF : (uint32_t)plan.tile * 128u);      // of both CTAs
            for (int step = 0; step < steps; ++step) {
                if (!poll(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag)) goto done;
                if (elect_one()) {
                    if (cta == 0) mbar_expect_tx(bar_full + 8 * ring.slot, bytes);
                    const uint32_t dst = smem0 + ring.slot * p.stage, other = dst + p.row_bytes, bar = leader_full + 8 * ring.slot;
                    if (GRAD && it.of_grad) {
                        const int v = it.piece * plan.piece + step * kHeadStep;
                        if (here) tma_load_2d_pair(dst, &tm_probs, bar, step * kHeadStep, row0);
                        tma_load_2d_pair(other, &tm_head_t, bar, other0, v);
                        tma_load_2d_pair(other + HL_HALF / 2, &tm_head_t, bar, other0 + 64, v);
                    } else {
                        if (here) tma_load_2d_pair(dst, of_rows, bar, step * kHeadStep, row0);
                        tma_load_2d_pair(other, &tm_head, bar, step * kHeadStep, other0);
                    }
                }
                __syncwarp();
                ring.advance(p.stages);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ products (leader)
        if (cta == 0) {
            // rows: contraction-contiguous, 128-byte swizzle, 8-row groups 1024 B apart; the head likewise for the logits, and for the gradient with
            // 64 features contiguous: 64-feature atoms 8192 B apart, groups of 8 entries 1024 B apart
            const uint64_t a_desc0 = smem_desc(smem0, 16, 1024, 2);
            const uint64_t b_logits = smem_desc(smem0 + p.row_bytes, 16, 1024, 2), b_grad = smem_desc(smem0 + p.row_bytes, 8192, 1024, 2);
            Ring ring;
            uint32_t n = 0;
            Item it;
            while (next(&it)) {
                const int steps = it.steps;
                const bool of_grad = GRAD && it.of_grad;
                const uint32_t idesc = instr_desc_pair(of_grad ? 256u : (uint32_t)plan.tile, 0u, of_grad ? 1u : 0u), b_k16 = of_grad ? 2048u >> 4 : 32u >> 4;
                const uint64_t b_desc0 = of_grad ? b_grad : b_logits;
                const uint32_t buffer = n & 1u, acc = tmem_base + buffer * 256u;
                if (!poll(bar_acc_empty + 8 * buffer, ((n >> 1) & 1u) ^ 1u, abort_flag)) goto done;
                tc_fence_after();
                for (int step = 0; step < steps; ++step) {
                    if (!poll(bar_full + 8 * ring.slot, ring.phase, abort_flag)) goto done;
                    tc_fence_after();
                    const uint32_t at = ring.slot * (p.stage >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t k = 0; k < kHeadStep / 16; ++k)
                            tc_mma_pair(acc, a_desc0 + at + k * 2, b_desc0 + at + k * b_k16, idesc, (uint32_t)(step > 0 || k > 0));
                        tc_commit_pair(bar_empty + 8 * ring.slot);
                        if (step + 1 == steps) tc_commit_pair(bar_acc_full + 8 * buffer);
                    }
                    __syncwarp();
                    ring.advance(p.stages);
                }
                ++n;
            }
        }
    } else if (warp >= HL_EPI_WARP0) {
        // ------------------------------------------------------------------ epilogue: a thread has one row
        const int quarter = warp & 3;
        const uint32_t leader_acc_empty = map_to_cta(bar_acc_empty, 0);
        uint8_t* slice = smem_gen + HL_OFF_SLICES + quarter * HL_SLICE;
        uint32_t n = 0;
        Item it;
        for (; next(&it); ++n) {
            const uint32_t buffer = n & 1u, taddr = tmem_base + buffer * 256u + ((uint32_t)(quarter * 32) << 16);
            const int row_w = it.block * kHeadTile + (int)cta * 128 + quarter * 32, row = row_w + lane;   // (of the buffers: row < p.padded)
            if (GRAD && it.of_grad) {
                // ---- a tile of the gradient's sums
                const int set = it.piece % plan.sums;
                const bool add = it.piece >= plan.sums;
                const unsigned* before = grads_done(p) + (size_t)(add ? it.q - plan.sums : it.q) * kHeadChunk + it.block_in_chunk;
                if (add && !poll_counter(before, COUNTS_PER_TILE * plan.feature_tiles, abort_flag)) break;
                if (!poll(bar_acc_full + 8 * buffer, (n >> 1) & 1u, abort_flag)) break;
                tc_fence_after();
                float* out = p.sums + ((size_t)set * p.padded + row_w) * plan.D;
                const int rows_here = n_rows - row_w;
#pragma unroll 1
                for (int idx = 0; idx < (row_w < n_rows ? 8 : 0); ++idx) {
                    const int c = it.tile * kHeadTile + 32 * idx + 4 * (lane & 7);
                    float4 old[8];
                    if (add) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int R = 4 * i + (lane >> 3);
                            old[i] = R < rows_here && c < plan.D ? __ldcg(reinterpret_cast<const float4*>(out + (size_t)R * plan.D + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                    }
                    uint32_t v[32];
                    tc_ld32(taddr + 32 * idx, v);
                    tc_wait_ld();
                    __syncwarp();                                      // the previous chunk has been read back
#pragma unroll
                    for (int c4 = 0; c4 < 8; ++c4)
                        *reinterpret_cast<uint4*>(slice + lane * 128 + ((c4 ^ (lane & 7)) << 4)) = make_uint4(v[4 * c4], v[4 * c4 + 1], v[4 * c4 + 2], v[4 * c4 + 3]);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int R = 4 * i + (lane >> 3);
                        float4 x = *reinterpret_cast<const float4*>(slice + R * 128 + (((lane & 7) ^ (R & 7)) << 4));
                        if (add) { x.x += old[i].x; x.y += old[i].y; x.z += old[i].z; x.w += old[i].w; }
                        if (R < rows_here && c < plan.D) __stcg(reinterpret_cast<float4*>(out + (size_t)R * plan.D + c), x);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(leader_acc_empty + 8 * buffer);
                publish(grads_done(p) + (size_t)it.q * kHeadChunk + it.block_in_chunk);
                continue;
            }
            // ---- a tile of logits
            const int v0 = it.piece * plan.piece + it.tile * plan.tile, valid = min(plan.V - v0, plan.tile), chunks = row_w < n_rows ? plan.tile / 32 : 0;
            const int label = row < n_rows ? __ldcg(p.label + row) - v0 : -1;
            const bool first = it.piece == 0 && it.tile == 0 && !p.again;
            float ref = 0.f;
            if (GRAD) {
                const int before = head_slot_before(plan, rows, it.q, it.block_in_chunk, active);
                if (before >= 0) {                                     // the slot's previous probabilities have been read
                    const unsigned* read = grads_done(p) + (size_t)before * kHeadChunk + it.block_in_chunk;
                    if (!poll_counter(read, COUNTS_PER_TILE * plan.feature_tiles, abort_flag)) break;
                }
                if (!first) {
                    if (!p.again && !poll_counter(ref_known(p) + it.block, COUNTS_PER_TILE, abort_flag)) break;
                    ref = __ldcg(p.ref + row);
                }
            }
            if (!poll(bar_acc_full + 8 * buffer, (n >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            if (GRAD && first) {
                // the others' alone: a label that is far above them would take the reference out of their reach
                float m = -INFINITY, mine = -INFINITY;
#pragma unroll 1
                for (int idx = 0; idx < chunks; ++idx) {
                    uint32_t v[32];
                    tc_ld32(taddr + 32 * idx, v);
                    tc_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float x = __uint_as_float(v[j]);
                        if (32 * idx + j == label) mine = x;
                        else if (32 * idx + j < valid) m = fmaxf(m, x);
                    }
                }
                if (m == -INFINITY) m = mine;
                ref = m == -INFINITY ? 0.f : fminf(m + REF_ABOVE, MOST);
                __stcg(p.ref + row, ref);
                publish(ref_known(p) + it.block);
            }
            float m = -INFINITY, s = 0.f;                              // the largest logit; the sum over the reference, or over m
            f2 rounded = make_f2(0.f, 0.f);                            // the sum of the probabilities as they are stored
            bf16* out = nullptr;
            if constexpr (GRAD)
                out = p.probs + it.tile * plan.tile +
                      ((size_t)((it.q % plan.ring) * plan.chunk_max + it.block_in_chunk) * kHeadTile + (int)cta * 128 + quarter * 32) * plan.piece;
            // 32 logits of the row; SPECIAL: the label or the vocabulary's end is among some row's
            auto chunk = [&](uint32_t (&v)[32], int idx, auto special) {
                constexpr bool SPECIAL = decltype(special)::value;
                float sum[2] = {0.f, 0.f};
                if constexpr (SPECIAL) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        if (32 * idx + j == label) __stcg(p.label_logit + row, __uint_as_float(v[j]));
                        if (32 * idx + j >= valid) v[j] = 0xFF800000u;           // -inf
                    }
                }
                float top = __uint_as_float(v[0]);
#pragma unroll
                for (int j = 1; j < 32; ++j) top = fmaxf(top, __uint_as_float(v[j]));
                const float to = fmaxf(m, top), base = GRAD ? ref : to == -INFINITY ? 0.f : to;
                if constexpr (!GRAD) s *= fast_exp2((m - base) * p.scale);
                m = to;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    float e = fast_exp2((__uint_as_float(v[j]) - base) * p.scale);
                    if (SPECIAL && 32 * idx + j == label) e = 0.f;
                    sum[j & 1] += e;
                    v[j] = __float_as_uint(e);
                }
                s += sum[0] + sum[1];
                if constexpr (GRAD) {
                    // by rows into the warp's slice, out of it so that four lanes have 64 bytes of a row
                    __syncwarp();
#pragma unroll
                    for (int c8 = 0; c8 < 4; ++c8) {
                        uint32_t o[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const __nv_bfloat162 pr = __floats2bfloat162_rn(__uint_as_float(v[c8 * 8 + 2 * j]), __uint_as_float(v[c8 * 8 + 2 * j + 1]));
                            o[j] = *reinterpret_cast<const uint32_t*>(&pr);
                            rounded = add2(rounded, unpack_bf16(o[j]));
                        }
                        *reinterpret_cast<uint4*>(slice + lane * 64 + ((c8 ^ ((lane >> 1) & 3)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int R = 8 * i + (lane >> 2);
                        const uint4 val = *reinterpret_cast<const uint4*>(slice + R * 64 + (((lane & 3) ^ ((R >> 1) & 3)) << 4));
                        __stcg(reinterpret_cast<uint4*>(out + (size_t)R * plan.piece + 32 * idx + 8 * (lane & 3)), val);
                    }
                }
            };
#pragma unroll 1
            for (int idx = 0; idx < chunks; ++idx) {
                uint32_t v[32];
                tc_ld32(taddr + 32 * idx, v);
                tc_wait_ld();
                const bool special = 32 * idx + 32 > valid || (label >= 32 * idx && label < 32 * idx + 32);
                if (__any_sync(0xFFFFFFFFu, special)) chunk(v, idx, std::true_type{});
                else chunk(v, idx, std::false_type{});
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(leader_acc_empty + 8 * buffer);
            const size_t stats = (size_t)row * head_div_up(plan.V, plan.tile) + v0 / plan.tile;
            __stcg(p.tile_stats + stats, make_float2(m, s));
            if constexpr (GRAD) __stcg(p.tile_rounded + stats, lo_of(rounded) + hi_of(rounded));
            if constexpr (GRAD) publish(logits_done(p) + (size_t)it.q * kHeadChunk + it.block_in_chunk);
        }
    }

done:
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {   // copies that may still be in flight land before the CTA's memory is released
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
        __syncthreads();
    }
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// Tokens that have a label become rows, in their order: place[t] (-1 without), the rows' labels, and, unless every token has one, the hidden states side
// by side.  A block takes 8 tokens at a time, a warp each, and counts the labels itself: those before its tokens and all of them.  The counters are set to zero.
// Every block reads all the labels; with more than 16384 tokens it takes 8 several times, so that this does not grow as the square of the tokens.
constexpr int PREP_TOKENS = 8, PREP_THREADS = 32 * PREP_TOKENS, PREP_BLOCKS = 2048;
__global__ void __launch_bounds__(PREP_THREADS)
head_prepare_kernel(int T, int V, int D, int copies, int turns, const int32_t* __restrict__ labels, const bf16* __restrict__ hidden, int* __restrict__ place,
                    int* __restrict__ row_label, bf16* __restrict__ rows, unsigned* __restrict__ counters, size_t counter_words) {
    __shared__ int parts[2][PREP_TOKENS];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t0 = blockIdx.x * turns * PREP_TOKENS;
    for (size_t i = 1 + blockIdx.x * PREP_THREADS + threadIdx.x; i < counter_words; i += (size_t)gridDim.x * PREP_THREADS) counters[i] = 0u;
    int before = 0, after = 0;                                         // labels of tokens before this warp's, and of the others
    for (int i = threadIdx.x; i < T; i += PREP_THREADS) {
        const int has = (unsigned)__ldg(labels + i) < (unsigned)V;
        before += i < t0 ? has : 0;
        after += i < t0 ? 0 : has;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
        after += __shfl_xor_sync(0xFFFFFFFFu, after, o);
    }
    if (lane == 0) { parts[0][warp] = before; parts[1][warp] = after; }
    __syncthreads();
    before = after = 0;
#pragma unroll
    for (int w = 0; w < PREP_TOKENS; ++w) { before += parts[0][w]; after += parts[1][w]; }
    const int all = before + after;
    if (t0 == 0 && threadIdx.x == 0) counters[0] = (unsigned)all;
    for (int turn = 0; turn < turns; ++turn) {
        const int first = t0 + turn * PREP_TOKENS, t = first + warp;
        const int label = lane < PREP_TOKENS && first + lane < T ? __ldg(labels + first + lane) : -1;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, (unsigned)label < (unsigned)V);
        const int at = (mask >> warp) & 1u ? before + __popc(mask & ((1u << warp) - 1u)) : -1, mine = __shfl_sync(0xFFFFFFFFu, label, warp);
        before += __popc(mask);
        if (lane == 0 && t < T) {
            place[t] = at;
            if (at >= 0) row_label[at] = mine;
        }
        if (at < 0 || (all == T && !copies)) continue;
        const uint4* src = reinterpret_cast<const uint4*>(hidden + (size_t)t * D);
        uint4* dst = reinterpret_cast<uint4*>(rows + (size_t)at * D);
#pragma unroll 8
        for (int c = lane; c < D / 8; c += 32) dst[c] = __ldg(src + c);
    }
}

// One block per token: its loss from the tiles' sums, and its row of the gradient from the pieces' sums, which are asked for first.
constexpr int FIN_THREADS = 256, FIN_AHEAD = 2;
struct MaxSum { float m, s, r; };             // r: the sum of the rounded terms, with the gradient
// Each thread's maximum and sum -> the block's (in a fixed order).
template <bool RESCALE>
__device__ __forceinline__ MaxSum block_max_sum(MaxSum v, float scale, float (*parts)[3]) {
    auto join = [&](MaxSum a, MaxSum b) {
        MaxSum r{fmaxf(a.m, b.m), a.s + b.s, a.r + b.r};
        if constexpr (RESCALE)                                         // (a sum over its own maximum; one without a term has none)
            r.s = (a.s == 0.f ? 0.f : a.s * fast_exp2((a.m - r.m) * scale)) + (b.s == 0.f ? 0.f : b.s * fast_exp2((b.m - r.m) * scale));
        return r;
    };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join(v, MaxSum{__shfl_xor_sync(0xFFFFFFFFu, v.m, o), __shfl_xor_sync(0xFFFFFFFFu, v.s, o), RESCALE ? 0.f : __shfl_xor_sync(0xFFFFFFFFu, v.r, o)});
    if ((threadIdx.x & 31) == 0) { parts[threadIdx.x >> 5][0] = v.m; parts[threadIdx.x >> 5][1] = v.s; parts[threadIdx.x >> 5][2] = v.r; }
    __syncthreads();
    v = MaxSum{parts[0][0], parts[0][1], parts[0][2]};
#pragma unroll
    for (int w = 1; w < FIN_THREADS / 32; ++w) v = join(v, MaxSum{parts[w][0], parts[w][1], parts[w][2]});
    return v;
}

template <bool GRAD>
__global__ void __launch_bounds__(FIN_THREADS)
head_finish_kernel(HeadParams p, const int* __restrict__ place, const bf16* __restrict__ head, const float* __restrict__ d_loss, float* __restrict__ loss,
                   bf16* __restrict__ d_hidden) {
    __shared__ float parts[FIN_THREADS / 32][3];
    pdl_launch_dependents();
    pdl_wait();
    if (p.again && __ldcg(p.counters + 3) == 0u) return;
    for (int t = blockIdx.x; t < p.tokens; t += gridDim.x) {
        const int row = __ldcg(place + t), D = p.plan.D, chunks = D / 8;
        uint4* out = GRAD ? reinterpret_cast<uint4*>(d_hidden + (size_t)t * D) : nullptr;
        if (row < 0) {
            if (p.again) continue;
            if (threadIdx.x == 0) loss[t] = 0.f;
            if (GRAD)
                for (int c = threadIdx.x; c < chunks; c += FIN_THREADS) out[c] = make_uint4(0, 0, 0, 0);
            continue;
        }
        if (p.again && __ldcg(to_do_again(p) + row / kHeadTile) == 0u) continue;
        // eight features of the row: the pieces' sums and the label's row of the head
        struct Chunk { float v[8]; uint4 w; };
        const uint4* w = GRAD ? reinterpret_cast<const uint4*>(head + (size_t)__ldcg(p.label + row) * D) : nullptr;
        const float* sums = GRAD ? p.sums + (size_t)row * D : nullptr;
        auto load = [&](int c) {
            Chunk x{};
            for (int k = 0; k < p.plan.sums; ++k) {
                const float4* from = reinterpret_cast<const float4*>(sums + (size_t)k * p.padded * D) + 2 * c;
                const float4 a = __ldcg(from), b = __ldcg(from + 1);
                x.v[0] += a.x; x.v[1] += a.y; x.v[2] += a.z; x.v[3] += a.w;
                x.v[4] += b.x; x.v[5] += b.y; x.v[6] += b.z; x.v[7] += b.w;
            }
            x.w = __ldg(w + c);
            return x;
        };
        Chunk ahead[FIN_AHEAD];
        if constexpr (GRAD) {
#pragma unroll
            for (int i = 0; i < FIN_AHEAD; ++i)
                if (threadIdx.x + i * FIN_THREADS < chunks) ahead[i] = load(threadIdx.x + i * FIN_THREADS);
        }
        const int tiles = head_div_up(p.plan.V, p.plan.tile);
        const float label_logit = __ldcg(p.label_logit + row), known_ref = GRAD ? __ldcg(p.ref + row) : 0.f;
        MaxSum v{-INFINITY, 0.f, 0.f};
        for (int i = threadIdx.x; i < tiles; i += FIN_THREADS) {
            const float2 stats = __ldcg(p.tile_stats + (size_t)row * tiles + i);
            const float m = stats.x, s = stats.y;
            if constexpr (GRAD) v = MaxSum{fmaxf(v.m, m), v.s + s, v.r + __ldcg(p.tile_rounded + (size_t)row * tiles + i)};
            else {
                const float to = fmaxf(v.m, m);
                v.s = (v.s == 0.f ? 0.f : v.s * fast_exp2((v.m - to) * p.scale)) + (s == 0.f ? 0.f : s * fast_exp2((m - to) * p.scale));
                v.m = to;
            }
        }
        v = block_max_sum<!GRAD>(v, p.scale, parts);
        const float ref = GRAD ? known_ref : v.m, others = v.s;
        const float at_label = (label_logit - ref) * p.scale, mine = fast_exp2(at_label), total = others + mine;
        if (threadIdx.x == 0) {
            // (a label that has most of the probability: the small loss from the small sum)
            float l = others <= mine ? log1pf(others / mine) : LN2 * (log2f(total) - at_label);
            if (!(total < INFINITY)) l = NAN;
            loss[t] = l;
            if (GRAD && !p.again && v.m - ref > REF_REACH) {
                p.counters[3] = 1u;
                to_do_again(p)[row / kHeadTile] = 1u;
                p.ref[row] = fminf(v.m, MOST);
            }
        }
        if constexpr (GRAD) {
            // The pieces' sums hold rounded probabilities.  They are given the weight that the unrounded ones have, which is what the label's row is subtracted
            // with: what all rows of the head have in common cancels to fp32's rounding.
            // (A label whose logit is +infinity: a probability of infinity / infinity.)
            const float f = d_loss[t], unit = total < INFINITY ? f / total : NAN, back = -unit * others, share = v.r > 0.f ? unit * (others / v.r) : unit;
            auto store = [&](int c, const Chunk& x) {
                const uint32_t lw[4] = {x.w.x, x.w.y, x.w.z, x.w.w};
                uint32_t o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const __nv_bfloat162 pr = __floats2bfloat162_rn(fmaf(share, x.v[2 * j], back * bf16_lo(lw[j])), fmaf(share, x.v[2 * j + 1], back * bf16_hi(lw[j])));
                    o[j] = f == 0.f ? 0u : *reinterpret_cast<const uint32_t*>(&pr);
                }
                out[c] = make_uint4(o[0], o[1], o[2], o[3]);
            };
#pragma unroll
            for (int i = 0; i < FIN_AHEAD; ++i)
                if (threadIdx.x + i * FIN_THREADS < chunks) store(threadIdx.x + i * FIN_THREADS, ahead[i]);
            for (int c = threadIdx.x + FIN_AHEAD * FIN_THREADS; c < chunks; c += FIN_THREADS) store(c, load(c));
        }
        __syncthreads();                                               // `parts` is written again
    }
}

// The waits' way out: a barrier that nobody arrives at, and a counter that nothing adds to, a warp each.
__device__ unsigned g_head_never = 0;
__global__ void __launch_bounds__(64)
head_wait_probe_kernel(int limit_us) {
    __shared__ uint64_t bar;
    __shared__ int flags[2][2];                                        // (one for each wait: neither ends because the other has)
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        flags[0][0] = flags[1][0] = 0;
        flags[0][1] = flags[1][1] = limit_us;
        mbar_init(smem_u32(&bar), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (warp == 0) (void)poll(smem_u32(&bar), 0u, flags[0]);
    else (void)poll_counter(&g_head_never, 1u, flags[1]);
}

}  // namespace

int launch_head_wait_probe(int limit_us, cudaStream_t st) {
    head_wait_probe_kernel<<<1, 64, 0, st>>>(limit_us);
    return cudaGetLastError() == cudaSuccess ? QLORA_OK : QLORA_ERR_CUDA;
}

size_t head_loss_workspace_bytes(int T, int V, int D, bool grad) { return head_layout(head_plan(T, V, D, grad ? 1 : 0), T).total; }

template <bool GRAD>
static int head_loss_impl(int T, int V, int D, const void* hidden, const void* head, const int32_t* labels, const float* d_loss, float* loss, void* d_hidden,
                          void* workspace, cudaStream_t st) {
    HeadParams p{};
    p.plan = head_plan(T, V, D, GRAD ? 1 : 0);
    const HeadLayout l = head_layout(p.plan, T);
    char* ws = static_cast<char*>(workspace);
    p.wait_limit_us = HL_WAIT_US;
    p.scale = LOG2E * (1.0f + CUT_OFF * (float)(D < CUT_OFF_LENGTH ? D : CUT_OFF_LENGTH));
    p.padded = (size_t)p.plan.blocks_max * kHeadTile;
    p.counters = reinterpret_cast<unsigned*>(ws + l.counters);
    p.label = reinterpret_cast<int*>(ws + l.label);
    p.ref = reinterpret_cast<float*>(ws + l.ref);
    p.label_logit = reinterpret_cast<float*>(ws + l.label_logit);
    p.tile_stats = reinterpret_cast<float2*>(ws + l.tile_stats);
    p.tile_rounded = reinterpret_cast<float*>(ws + l.tile_rounded);
    p.probs = reinterpret_cast<bf16*>(ws + l.probs);
    p.sums = reinterpret_cast<float*>(ws + l.sums);
    int* place = reinterpret_cast<int*>(ws + l.place);
    bf16* rows = reinterpret_cast<bf16*>(ws + l.rows);

    p.tokens = T;
    p.copies = hidden == d_hidden;                                     // (the second launch still reads them)
    CUtensorMap tx, tr, th, tt{}, tp{};
    const CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const uint32_t rows_box = T < 128 ? (uint32_t)(T + 7) / 8 * 8 : 128;
    p.row_bytes = rows_box * 128;
    p.stage = p.row_bytes + HL_HALF;
    p.stages = HL_RING / p.stage < HL_MAX_STAGES ? HL_RING / p.stage : HL_MAX_STAGES;
    if (!make_map_2d(&tx, type, 2, hidden, (uint64_t)D, (uint64_t)T, 64, rows_box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_2d(&tr, type, 2, rows, (uint64_t)D, p.padded, 64, rows_box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_2d(&th, type, 2, head, (uint64_t)D, (uint64_t)V, 64, (uint32_t)p.plan.tile / 2, CU_TENSOR_MAP_SWIZZLE_128B))
        return QLORA_ERR_CUDA;
    if (GRAD && (!make_map_2d(&tt, type, 2, head, (uint64_t)D, (uint64_t)V, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B) ||
                 !make_map_2d(&tp, type, 2, p.probs, (uint64_t)p.plan.piece, (uint64_t)p.plan.ring * p.plan.chunk_max * kHeadTile, 64, rows_box, CU_TENSOR_MAP_SWIZZLE_128B)))
        return QLORA_ERR_CUDA;
    static SmemLimit limit;
    auto kern = head_loss_kernel<GRAD>;
    if (!limit.raise(kern, HL_SMEM)) return QLORA_ERR_CUDA;
    const int turns = (T + PREP_TOKENS * PREP_BLOCKS - 1) / (PREP_TOKENS * PREP_BLOCKS);
    if (launch_pdl(head_prepare_kernel, dim3((T + turns * PREP_TOKENS - 1) / (turns * PREP_TOKENS)), dim3(PREP_THREADS), 0, st, 1, T, V, D, p.copies, turns, labels, (const bf16*)hidden, place,
                   const_cast<int*>(p.label), rows, p.counters, l.counter_words) != cudaSuccess)
        return QLORA_ERR_CUDA;
    const long long items = head_rows(p.plan, T).total;
    const int pairs = (int)(items < sm_count() / 2 ? items : sm_count() / 2);
    for (p.again = 0; p.again < (GRAD ? 2 : 1); ++p.again) {
        if (launch_pdl(kern, dim3(2 * pairs), dim3(HL_THREADS), HL_SMEM, st, 1, tx, tr, th, tt, tp, p) != cudaSuccess) return QLORA_ERR_CUDA;
        const int blocks = p.again && T > 4 * sm_count() ? 4 * sm_count() : T;
        if (launch_pdl(head_finish_kernel<GRAD>, dim3(blocks), dim3(FIN_THREADS), 0, st, 1, p, place, (const bf16*)head, d_loss, loss, (bf16*)d_hidden) != cudaSuccess)
            return QLORA_ERR_CUDA;
    }
    return QLORA_OK;
}

int launch_head_loss(int T, int V, int D, const void* hidden, const void* head, const int32_t* labels, const float* d_loss, float* loss, void* d_hidden,
                     void* workspace, cudaStream_t st) {
    return d_hidden != nullptr ? head_loss_impl<true>(T, V, D, hidden, head, labels, d_loss, loss, d_hidden, workspace, st)
                               : head_loss_impl<false>(T, V, D, hidden, head, labels, nullptr, loss, nullptr, workspace, st);
}

int read_head_status(unsigned int* out, int clear) {
    unsigned int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_head_status, sizeof(v)) != cudaSuccess) return QLORA_ERR_CUDA;
    if (clear && v != 0) {
        const unsigned int zero = 0;
        if (cudaMemcpyToSymbol(g_head_status, &zero, sizeof(zero)) != cudaSuccess) return QLORA_ERR_CUDA;
    }
    *out = v;
    return QLORA_OK;
}

}  // namespace qlora
