"""The order of the work behind the head's cross entropy, checked on the CPU: every tile once, and nothing waits for what is claimed after it."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "head_plan.h"
using namespace qlora;
struct Out { int blocks_max, chunk_max, tile, piece, pieces, features, ring, sums, blocks, chunk, chunks, all_pieces, lead; long long total; };
extern "C" void plan(int T, int V, int D, int grad, int rows, Out* o) {
    const HeadPlan p = head_plan(T, V, D, grad);
    const HeadRows r = head_rows(p, rows);
    *o = Out{p.blocks_max, p.chunk_max, p.tile, p.piece, p.pieces, p.feature_tiles, p.ring, p.sums, r.blocks, r.chunk, r.chunks, r.all_pieces, r.lead, r.total};
}
extern "C" void items(int T, int V, int D, int grad, int rows, long long n, int* out) {
    const HeadPlan p = head_plan(T, V, D, grad);
    const HeadRows r = head_rows(p, rows);
    for (long long i = 0; i < n; ++i) {
        const HeadItem it = head_item(p, r, i);
        const int v[6] = {it.of_grad, it.q, it.piece, it.block_in_chunk, it.block, it.tile};
        for (int k = 0; k < 6; ++k) out[6 * i + k] = v[k];
    }
}
extern "C" unsigned long long bytes(int T, int V, int D, int grad) { return head_layout(head_plan(T, V, D, grad), T).total; }
extern "C" unsigned long long words(int T, int V, int D, int grad) { return head_layout(head_plan(T, V, D, grad), T).counter_words; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("head_plan")
    (d / "p.cpp").write_text(SOURCE)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2306_08162_b200", "csrc"), str(d / "p.cpp"), "-o",
                    str(d / "p.so")], check=True)
    lib = ctypes.CDLL(str(d / "p.so"))
    lib.bytes.restype = lib.words.restype = ctypes.c_ulonglong
    return lib


class Out(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in "blocks_max chunk_max tile piece pieces features ring sums blocks chunk chunks all_pieces lead".split()] + [("total", ctypes.c_longlong)]


SHAPES = [(T, V, D, rows) for T, rows in ((1, 1), (16, 9), (256, 256), (257, 257), (600, 600), (2048, 2048), (2049, 2049), (2305, 2048), (2305, 17), (8192, 8192), (5000, 4100), (9000, 0))
          for V, D in ((1, 64), (255, 520), (4096, 4096), (4097, 64), (9000, 1000), (32000, 4096), (50021, 2568))]


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("T,V,D,rows", SHAPES)
def test_every_tile_once_and_in_an_order_without_circles(lib, T, V, D, rows, grad):
    o = Out()
    lib.plan(T, V, D, grad, rows, ctypes.byref(o))
    assert o.piece % 256 == 0 and o.piece * o.pieces >= V > o.piece * (o.pieces - 1) and o.chunk <= o.chunk_max <= 8 and o.chunk * o.chunks >= o.blocks
    flat = (ctypes.c_int * (6 * max(o.total, 1)))()
    lib.items(T, V, D, grad, rows, ctypes.c_longlong(o.total), flat)
    items = [tuple(flat[6 * i:6 * i + 6]) for i in range(o.total)]
    entries = lambda piece: min(o.piece, V - piece * o.piece)  # noqa: E731
    real = [it for it in items if it[4] < o.blocks and (it[0] or it[5] * o.tile < entries(it[2]))]
    logits, grads = [it for it in real if not it[0]], [it for it in real if it[0]]
    assert sorted((it[4], it[2] * (o.piece // o.tile) + it[5]) for it in logits) == [(b, t) for b in range(o.blocks) for t in range(-(-V // o.tile))]
    if not grad:
        assert not grads
        return
    assert sorted((it[4], it[2], it[5]) for it in grads) == [(b, p, f) for b in range(o.blocks) for p in range(o.pieces) for f in range(o.features)]
    at = {it: i for i, it in enumerate(real)}
    last_logits, last_grad = {}, {}
    for it, i in at.items():
        key = (it[1], it[3])
        (last_grad if it[0] else last_logits)[key] = i
    first = {it[4]: i for it, i in at.items() if not it[0] and it[2] == 0 and it[5] == 0}
    for it, i in at.items():
        assert 0 <= it[1] < -(-o.blocks_max // 8) * o.pieces and 0 <= it[3] < 8                    # inside the counters
        if it[0]:
            assert last_logits[(it[1], it[3])] < i                                              # its probabilities
            if it[2] >= o.sums:
                assert last_grad[(it[1] - o.sums, it[3])] < i                                   # the sums it adds to
        else:
            assert first[it[4]] <= i                                                            # the reference
            before = it[1] - o.ring
            if before >= 0 and (before // o.pieces) * o.chunk + it[3] < o.blocks:
                assert last_grad[(before, it[3])] < i                                           # who read the slot before


def test_the_workspace_does_not_hold_the_logits(lib):
    assert lib.bytes(8192, 128000, 4096, 1) < 8192 * 128000 * 2 // 4
    for T, V, D in ((1, 1, 64), (300, 50021, 1000), (2048, 32000, 4096)):
        for grad in (0, 1):
            assert lib.bytes(T, V, D, grad) % 1024 == 0 and lib.bytes(T, V, D, grad) > 4 * lib.words(T, V, D, grad)
