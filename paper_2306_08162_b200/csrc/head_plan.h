// How the head's cross entropy is cut into items of work, on the host and on the device (plain C++: the tests build it for the CPU).
//
// The tokens that have a label are counted as rows, in blocks of 256; up to 8 blocks are a chunk, which goes through the vocabulary piece by piece.
// A piece q (counted over all chunks) is two sets of items: its logits, tiles of 256 rows x 256 vocabulary entries, and its part of the gradient, tiles of 256 rows x 256
// hidden features that add the piece's part to fp32 sums.  Items are claimed in one order: the logits of the first `lead`
// pieces, then the logits of piece q + lead and the gradient of piece q in turn, so that what an item waits for was claimed before it.
#pragma once
#include <stddef.h>

#ifdef __CUDACC__
#define QLORA_HD __host__ __device__ __forceinline__
#else
#define QLORA_HD inline
#endif

namespace qlora {

constexpr int kHeadTile = 256, kHeadStep = 64;   // rows and features of a tile, entries at most; contraction elements of a step
constexpr int kHeadChunk = 8;                    // row blocks of a chunk
constexpr int kHeadPairs = 74;                   // pairs of SMs
constexpr int kHeadPiece = 4096;                 // vocabulary entries of a piece at most

QLORA_HD int head_div_up(int a, int b) { return (a + b - 1) / b; }

struct HeadPlan {
    int V, D, grad;
    int blocks_max;                              // row blocks that the buffers hold (all tokens)
    int chunk_max;                               // row blocks of a chunk at most
    int tile;                                    // entries of a tile of logits (with 128 for few rows, whose time is that of reading the head: 58 -> 67 us)
    int piece, pieces, feature_tiles;            // entries of a piece (a multiple of 256); pieces; tiles across the hidden features
    int ring;                                    // pieces whose probabilities are kept at a time
    int sums;                                    // sets of fp32 sums: piece p adds to set p % sums
};

inline HeadPlan head_plan(int T, int V, int D, int grad) {
    HeadPlan p;
    p.V = V; p.D = D; p.grad = grad;
    p.blocks_max = head_div_up(T, kHeadTile);
    p.chunk_max = p.blocks_max < kHeadChunk ? p.blocks_max : kHeadChunk;
    p.tile = kHeadTile;
    p.feature_tiles = head_div_up(D, kHeadTile);
    const int tiles = p.chunk_max * p.feature_tiles;
    // Pieces: of 4096 entries, or shorter ones where the gradient would not give every pair an item.  The cost of a
    // choice, in steps: waves times an item's steps and what it takes beside them, and the sets of sums that are added up in the end.
    auto cut = [&](int n) {
        p.piece = head_div_up(head_div_up(V, n), kHeadTile) * kHeadTile;
        p.pieces = head_div_up(V, p.piece);
    };
    const int least = head_div_up(V, kHeadPiece);
    int best = least;
    if (grad && tiles * least < kHeadPairs) {
        double lowest = 1e300;
        for (int n = least; n <= least + 255 && n <= head_div_up(V, kHeadTile); ++n) {
            cut(n);
            const double cost = (double)head_div_up(tiles * p.pieces, kHeadPairs) * (p.piece / kHeadStep + 6) + (double)p.pieces * T * D * 2e-6;
            if (cost < lowest) { lowest = cost; best = n; }
        }
    }
    cut(best);
    // 48 MB of probabilities (what stays in L2), three pieces at least: one being read, one written, one between
    const long long slot = 2ll * p.chunk_max * kHeadTile * p.piece;
    const long long fit = (48ll << 20) / slot;
    const int most = p.pieces * head_div_up(p.blocks_max, kHeadChunk);
    p.ring = fit < 3 ? 3 : fit < most ? (int)fit : most;
    // as many sets of sums as there are pieces under way at a time where there are few tiles
    p.sums = tiles >= 128 ? 1 : head_div_up(128, tiles);
    if (p.sums > p.pieces) p.sums = p.pieces;
    return p;
}

// What the number of rows that have a label decides.
struct HeadRows {
    int blocks, chunk, chunks, all_pieces, lead, logit_items, grad_items;
    long long total;
};

QLORA_HD HeadRows head_rows(const HeadPlan& p, int rows) {
    HeadRows r;
    r.blocks = head_div_up(rows, kHeadTile);
    r.chunks = head_div_up(r.blocks, kHeadChunk);
    r.chunk = r.chunks > 0 ? head_div_up(r.blocks, r.chunks) : 0;
    r.all_pieces = r.chunks * p.pieces;
    r.logit_items = r.chunk * (p.piece / p.tile);
    r.grad_items = p.grad ? r.chunk * p.feature_tiles : 0;
    // (the logits of piece q write where those of q - ring were: their gradient has to be claimed before, so lead < ring)
    r.lead = p.grad && r.all_pieces > p.ring ? (p.ring > 2 ? p.ring - 2 : 1) : r.all_pieces;
    r.total = (long long)r.all_pieces * (r.logit_items + r.grad_items);
    return r;
}

struct HeadItem { int of_grad, q, piece, block_in_chunk, block, tile; };   // tile: of the piece's entries, or of the features

QLORA_HD HeadItem head_item(const HeadPlan& p, const HeadRows& r, long long index) {
    HeadItem it;
    int i;
    const long long ahead = (long long)r.lead * r.logit_items, pair = r.logit_items + r.grad_items;
    if (index < ahead) {
        it.of_grad = 0;
        it.q = (int)(index / r.logit_items);
        i = (int)(index % r.logit_items);
    } else if (index - ahead < (r.all_pieces - r.lead) * pair) {
        const long long at = index - ahead;
        it.q = (int)(at / pair);
        i = (int)(at % pair);
        it.of_grad = i >= r.logit_items;
        if (it.of_grad) i -= r.logit_items;
        else it.q += r.lead;
    } else {
        const long long at = index - ahead - (r.all_pieces - r.lead) * pair;
        it.of_grad = 1;
        it.q = r.all_pieces - r.lead + (int)(at / r.grad_items);
        i = (int)(at % r.grad_items);
    }
    it.piece = it.q % p.pieces;
    it.block_in_chunk = i % r.chunk;
    it.block = it.q / p.pieces * r.chunk + it.block_in_chunk;
    it.tile = i / r.chunk;
    return it;
}

// The last piece before q whose probabilities lay where those of (q, block_in_chunk) go, or -1: its gradient has to be through before they are written.  Blocks
// of rows that take no part (the last chunk's missing ones; in the second launch those that are not done again) wrote and read nothing, so the one
// before them is who is waited for; it waited for the one before itself.
template <typename Active>
QLORA_HD int head_slot_before(const HeadPlan& p, const HeadRows& r, int q, int block_in_chunk, const Active& active) {
    for (int before = q - p.ring; before >= 0; before -= p.ring)
        if (active(before / p.pieces * r.chunk + block_in_chunk)) return before;
    return -1;
}

QLORA_HD int head_piece_entries(const HeadPlan& p, int piece) { return p.V - piece * p.piece < p.piece ? p.V - piece * p.piece : p.piece; }

// The workspace, in bytes from its beginning.
struct HeadLayout {
    size_t place, label, ref, label_logit, tile_stats, tile_rounded, rows, probs, sums, counters;
    size_t counter_words, total;
};

inline HeadLayout head_layout(const HeadPlan& p, int T) {
    HeadLayout l;
    size_t at = 0;
    const size_t padded = (size_t)p.blocks_max * kHeadTile, tiles = (size_t)head_div_up(p.V, p.tile);
    const int chunks = head_div_up(p.blocks_max, kHeadChunk);
#define QLORA_TAKE(name, bytes) l.name = at; at += ((size_t)(bytes) + 1023) / 1024 * 1024
    // [0] rows, [1] claimed, [2] claimed again, [3] anything to do again; per block: reference known, to do again; twice per piece and block: logits, gradient
    l.counter_words = 4 + 2 * (size_t)p.blocks_max + 4 * (size_t)chunks * p.pieces * kHeadChunk;
    QLORA_TAKE(counters, l.counter_words * 4);
    QLORA_TAKE(place, (size_t)T * 4);
    QLORA_TAKE(label, padded * 4);
    QLORA_TAKE(ref, padded * 4);
    QLORA_TAKE(label_logit, padded * 4);
    QLORA_TAKE(tile_stats, tiles * padded * 8);
    QLORA_TAKE(tile_rounded, p.grad ? tiles * padded * 4 : 0);
    QLORA_TAKE(rows, padded * p.D * 2);
    QLORA_TAKE(probs, p.grad ? (size_t)p.ring * p.chunk_max * kHeadTile * p.piece * 2 : 0);
    QLORA_TAKE(sums, p.grad ? (size_t)p.sums * padded * p.D * 4 : 0);
#undef QLORA_TAKE
    l.total = at;
    return l;
}

}  // namespace qlora
