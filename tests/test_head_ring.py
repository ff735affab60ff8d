"""The ring of probabilities behind the head's gradient where only some blocks of rows take part (the second launch), checked on the CPU: what is written
waits for the last one that read the same place, and that one was claimed before it."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "head_plan.h"
using namespace qlora;
struct Out { int piece, pieces, tile, features, ring, blocks, chunk, all_pieces; long long total; };
extern "C" void plan(int T, int V, int D, int rows, Out* o) {
    const HeadPlan p = head_plan(T, V, D, 1);
    const HeadRows r = head_rows(p, rows);
    *o = Out{p.piece, p.pieces, p.tile, p.feature_tiles, p.ring, r.blocks, r.chunk, r.all_pieces, r.total};
}
extern "C" void items(int T, int V, int D, int rows, long long n, int* out) {
    const HeadPlan p = head_plan(T, V, D, 1);
    const HeadRows r = head_rows(p, rows);
    for (long long i = 0; i < n; ++i) {
        const HeadItem it = head_item(p, r, i);
        const int v[6] = {it.of_grad, it.q, it.piece, it.block_in_chunk, it.block, it.tile};
        for (int k = 0; k < 6; ++k) out[6 * i + k] = v[k];
    }
}
extern "C" int before(int T, int V, int D, int rows, int q, int block_in_chunk, const unsigned char* part) {
    const HeadPlan p = head_plan(T, V, D, 1);
    const HeadRows r = head_rows(p, rows);
    return head_slot_before(p, r, q, block_in_chunk, [&](int block) { return block < r.blocks && part[block] != 0; });
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("head_ring")
    (d / "p.cpp").write_text(SOURCE)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2306_08162_b200", "csrc"), str(d / "p.cpp"), "-o",
                    str(d / "p.so")], check=True)
    return ctypes.CDLL(str(d / "p.so"))


class Out(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in "piece pieces tile features ring blocks chunk all_pieces".split()] + [("total", ctypes.c_longlong)]


CASES = [(8192, 32000, 4096, 8192, {0, 16}), (8192, 32000, 4096, 8192, {1, 17}), (6144, 32000, 4096, 6144, {3, 19}), (8192, 128000, 4096, 8192, {0, 16, 24}), (6144, 50021, 2568, 6144, {2, 18}),
         (5000, 50021, 2568, 5000, {0, 14}), (16384, 9000, 512, 16384, {5, 21, 45, 61}), (20000, 4000, 64, 19000, {0, 24, 72}), (9000, 12300, 264, 8000, {0, 1, 9, 31}), (1100, 9000, 128, 1100, {1, 2}),
         (8192, 32000, 512, 8192, set(range(32))), (8192, 32000, 512, 8192, set())]


@pytest.mark.parametrize("T,V,D,rows,part", CASES)
def test_what_is_written_waits_for_the_last_reader(lib, T, V, D, rows, part):
    o = Out()
    lib.plan(T, V, D, rows, ctypes.byref(o))
    assert all(b < o.blocks for b in part)
    flat = (ctypes.c_int * (6 * o.total))()
    lib.items(T, V, D, rows, ctypes.c_longlong(o.total), flat)
    entries = lambda piece: min(o.piece, V - piece * o.piece)  # noqa: E731
    claimed = [tuple(flat[6 * i:6 * i + 6]) for i in range(o.total)]
    claimed = [it for it in claimed if it[4] in part and (it[0] or it[5] * o.tile < entries(it[2]))]
    last_grad = {(it[1], it[3]): i for i, it in enumerate(claimed) if it[0]}         # by piece and block of its chunk
    mask = (ctypes.c_ubyte * max(o.blocks, 1))(*[b in part for b in range(o.blocks)])
    readers = {}                                                                     # by place in the ring: the pieces that lay there, in order
    for q, k in sorted(last_grad):
        readers.setdefault((q % o.ring, k), []).append(q)
    waited = 0
    for i, (of_grad, q, _, k, _, _) in enumerate(claimed):
        if of_grad:
            continue
        mine = readers[(q % o.ring, k)]
        want = mine[mine.index(q) - 1] if mine.index(q) > 0 else -1
        assert lib.before(T, V, D, rows, q, k, mask) == want
        if want >= 0:
            waited += 1
            assert last_grad[(want, k)] < i
    if len({b // o.chunk for b in part}) > 1 and o.all_pieces > o.ring:
        assert waited > 0
