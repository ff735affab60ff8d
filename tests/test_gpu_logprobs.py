"""Parity of the log-probability kernels with the 64-bit oracle (needs a B200).

Tolerances.  The kernels work in fp32 (u = 2^-24) with exponentials of relative error 2^-21 at most.  d = c (z - max) carries a relative
error of 3u, so exp(d) one of 3u|d| (at most 2u of the sum, since |d| e^d < 0.4) + 2^-21; a sum of V positive terms is formed along chains of at
most V / 256 + 40 additions, one u each.  So log s is off by at most S = (V / 256 + 64) u, a log probability by S + 4u |log p|, and the
entropy log s - (sum e d) / s by S + (S + 8u) times the mean of |d|, which is at most log V + |log p_max| + H: 24 covers it for the logits here.
Gradients: p is off by (S + 4u (16 + |log p|)) relatively, the result is rounded once to its type (half a step)."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from oracle import qlora_oracle as orc
from gpu_util import to_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def chain(V):
    return (V / 256 + 64) * U


def make(T, V, dtype, seed, ld=None, offset=0, spread=3.0):
    """Logits [T, V] in a buffer with other numbers (NaN) around the rows; the view begins `offset` elements in."""
    ld = V if ld is None else ld
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((T * ld + 64,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    z = buf[offset:offset + T * ld].view(T, ld)[:, :V]
    z.copy_(torch.randn((T, V), device="cuda", generator=gen) * spread)
    tokens = torch.randint(0, V, (T,), device="cuda", generator=gen).int()
    return z, tokens


def forward(z, tokens, c, k, only=None):
    T = z.shape[0]
    nan = float("nan")
    out = dict(logprobs=torch.full((T,), nan, device="cuda"), entropy=torch.full((T,), nan, device="cuda"), stats=torch.full((T, 3), nan, device="cuda"),
               top_ids=torch.full((T, k), -7, dtype=torch.int32, device="cuda") if k else None,
               top_logprobs=torch.full((T, k), nan, device="cuda") if k else None)
    if only is not None:
        out = {key: v if key in only else None for key, v in out.items()}
    ql.qlora_token_logprobs(z, tokens, c, out["logprobs"], entropy=out["entropy"], top_ids=out["top_ids"], top_logprobs=out["top_logprobs"], stats=out["stats"])
    return out


def close(got, want, absolute, relative=4 * U):
    got, want = to_f64(got), np.asarray(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))          # infinities and NaN where they belong
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= absolute + relative * np.abs(want)
    assert (same | near).all(), float(np.nanmax(np.abs(got - want)))


def check_forward(z, tokens, c, k):
    V = z.shape[1]
    out = forward(z, tokens, c, k)
    want = orc.token_logprobs(to_f64(z), tokens.cpu().numpy() if tokens is not None else None, c, k)
    close(out["logprobs"], want["logprobs"], chain(V))
    close(out["entropy"], want["entropy"], 25 * chain(V))
    assert torch.equal(out["stats"][:, 2].nan_to_num(-1.0), out["entropy"].nan_to_num(-1.0))
    m = to_f64(out["stats"][:, 0])
    assert (m == want["stats"][:, 0])[~np.isnan(m)].all() and (np.isnan(m) == np.isnan(want["stats"][:, 0])).all()
    close(out["stats"][:, 1], want["stats"][:, 1], chain(V))
    if k:
        assert np.array_equal(out["top_ids"].cpu().numpy(), want["top_ids"])
        close(out["top_logprobs"], want["top_logprobs"], chain(V))
    return out, want


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,V,k", [(1, 1, 1), (1, 32000, 20), (3, 7, 7), (2, 8, 0), (5, 255, 64), (2, 256, 1), (1, 257, 5), (4, 1000, 32), (9, 4097, 20),
                                   (150, 2053, 3), (17, 32000, 5), (2, 50021, 64), (1, 128000, 20), (300, 515, 33), (40, 16001, 64),
                                   (2500, 70, 7), (1900, 1031, 20), (1300, 8200, 64), (1000, 10007, 0),
                                   (3001, 331, 32), (6100, 70, 1), (160, 20011, 64), (1000, 16390, 31)])
def test_rows_of_every_length(T, V, k, dtype):
    z, tokens = make(T, V, dtype, seed=T + V + k)
    if T > 2:
        tokens[1], tokens[2] = -1, V                                 # outside the vocabulary
    check_forward(z, tokens, 1.0, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,ld,offset", [(4097, 4097, 0), (4097, 4097, 1), (1000, 1003, 5), (4096, 4160, 8), (513, 520, 3), (3, 5, 2), (32001, 32064, 0)])
def test_rows_that_lie_apart_and_begin_anywhere(V, ld, offset, dtype):
    """NaN between the rows and around them must not get into any row."""
    z, tokens = make(6, V, dtype, seed=V + ld, ld=ld, offset=offset)
    check_forward(z, tokens, 0.8, min(V, 9))


@pytest.mark.parametrize("c", [0.05, 0.7, 1.9, 30.0])
def test_temperatures(c):
    z, tokens = make(6, 3001, "bf16", seed=3)
    check_forward(z, tokens, c, 12)


@pytest.mark.parametrize("T", [1, 5, 200])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_masked_rows(dtype, T):
    """Entries ruled out by -inf or by the type's lowest value: most of a row, all but one, all; the chosen token among them; fewer entries
    left than alternatives asked for."""
    V, k = 3000, 20
    z, tokens = make(T, V, dtype, seed=11, ld=3008)
    low = torch.finfo(DTYPES[dtype]).min
    masks = [(slice(0, 0), 0.0), (slice(5, V), float("-inf")), (slice(0, V), float("-inf")), (slice(0, V), low), (slice(7, V), low)]
    for t in range(T):
        where, value = masks[(t + (2 if T == 1 else 0)) % 5]
        z[t, where] = value
        if t % 5 == 1:
            tokens[t] = 2900                                         # a token that is ruled out: -inf
    check_forward(z, tokens, 1.0, k)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_a_distribution_stay_by_themselves(bad, dtype):
    z, tokens = make(5, 2500, dtype, seed=13)
    z[1, 1234] = bad
    z[3, 0] = bad
    z[3, 2499] = float("nan")
    tokens[1] = -1
    out, _ = check_forward(z, tokens, 1.0, 6)
    assert torch.isfinite(out["logprobs"][[0, 2, 4]]).all() and torch.isnan(out["entropy"][[1, 3]]).all() and out["logprobs"][1] == 0


@pytest.mark.parametrize("V,k", [(5000, 64), (32000, 20), (700, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ties_and_orders(V, k, dtype):
    """Constant rows, few distinct values, ascending and descending rows, the largest at the end of a row, in a cluster, in one column of a
    regular pattern, zeros of both signs: equal logits come in the order of their places."""
    T = 9
    z, tokens = make(T, V, dtype, seed=V)
    j = torch.arange(V, device="cuda")
    z[0] = 1.5
    z[1] = (j % 3).to(z.dtype)
    z[2] = (j.float() / V * 4).to(z.dtype)
    z[3] = (-j.float() / V * 4).to(z.dtype)
    z[4, V - 70:] = 20.0
    z[5, 300:500] = 20.0 + (j[:200] % 7).to(z.dtype)
    z[6] = ((j % 256) == 17).to(z.dtype) * 5 + ((j % 2048) < 8).to(z.dtype)
    z[7] = torch.where(j % 2 == 0, -0.0, 0.0).to(z.dtype)
    z[8] = float("-inf")
    z[8, V - 3:] = 0.5
    check_forward(z, tokens, 1.0, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,k", [(3100, 1000, 20), (3100, 1501, 32), (170, 7000, 20), (170, 12001, 64), (170, 30000, 20), (160, 60011, 33), (460, 40000, 33), (20, 40000, 64)])
def test_odd_rows_among_many(T, V, k, dtype):
    """The rows of the tests above among as many others as make every way of sharing rows out take them: each with the oracle, the others with
    themselves in a batch where the odd rows are not."""
    z, tokens = make(T, V, dtype, seed=T + V, ld=V + 3)
    plain = forward(z, tokens, 1.0, k)                               # (the same memory: the order of a sum goes with where the row begins)
    j = torch.arange(V, device="cuda")
    odd = torch.arange(0, 14, device="cuda") * (T // 14)
    low, inf = torch.finfo(z.dtype).min, float("inf")
    z[odd[0]] = 1.5
    z[odd[1]] = (j % 3).to(z.dtype)
    z[odd[2]] = -inf
    z[odd[3]] = low
    z[odd[4], 5:] = -inf
    z[odd[5], 7:] = low
    z[odd[6], : V - 3] = -inf
    z[odd[7], V // 2] = float("nan")
    z[odd[8], V - 1] = inf
    z[odd[9], V - 70:] = 20.0
    z[odd[10], 300:600] = 20.0 + (j[:300] % 7).to(z.dtype)
    z[odd[11]] = torch.where(j % 2 == 0, -0.0, 0.0).to(z.dtype)
    z[odd[12], ::8] = 9.0
    z[odd[13]] = ((j % 2048) < 8).to(z.dtype)
    out = forward(z, tokens, 1.0, k)
    check = {key: v[odd] for key, v in out.items()}
    want = orc.token_logprobs(to_f64(z[odd]), tokens[odd].cpu().numpy(), 1.0, k)
    close(check["logprobs"], want["logprobs"], chain(V))
    close(check["entropy"], want["entropy"], 25 * chain(V))
    assert np.array_equal(check["top_ids"].cpu().numpy(), want["top_ids"])
    close(check["top_logprobs"], want["top_logprobs"], chain(V))
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[odd] = False
    for key in out:
        assert torch.equal(out[key][others], plain[key][others]), key


def test_large_logits_keep_their_differences():
    """Logits of several thousand: the statistics are relative to the row's maximum, so nothing is lost."""
    z, tokens = make(4, 9000, "fp32", seed=19)
    z += torch.tensor([[3e4], [-3e4], [1e30], [0.0]], device="cuda")
    check_forward(z, tokens, 1.0, 5)


def test_each_output_alone_and_none_at_all():
    z, tokens = make(7, 1000, "bf16", seed=23)
    full = forward(z, tokens, 1.0, 4)
    for only in (("logprobs",), ("entropy",), ("stats",), ("top_ids",), ("top_logprobs",), ("entropy", "top_ids")):
        got = forward(z, tokens if "logprobs" in only else None, 1.0, 4 if any(o.startswith("top") for o in only) else 0, only=only)
        for name in only:
            assert torch.equal(got[name], full[name]), name
    with pytest.raises(ql.QloraError) as e:
        forward(z, tokens, 1.0, 0, only=())
    assert e.value.status == -1
    empty = torch.empty((0, 1000), dtype=torch.bfloat16, device="cuda")
    ql.qlora_token_logprobs(empty, torch.empty(0, dtype=torch.int32, device="cuda"), 1.0, torch.empty(0, device="cuda"))


def test_same_bits_alone_and_in_company():
    """A row's numbers do not depend on the rows around it where the call takes the same way, and never on the run."""
    z, tokens = make(300, 4000, "bf16", seed=29)
    a, b = forward(z, tokens, 1.0, 8), forward(z, tokens, 1.0, 8)
    for key in a:
        assert torch.equal(a[key], b[key]), key
    one = forward(z[17:18], tokens[17:21][:1].clone(), 1.0, 8)
    assert torch.equal(one["top_ids"][0], a["top_ids"][17])
    close(one["logprobs"], to_f64(a["logprobs"][17:18]), 2 * chain(4000))


# ------------------------------------------------------------------------------------------------------ gradient

def check_backward(z, tokens, c, gl, gh, in_place=False, out=None):
    """Against the oracle's formula; what lies between the rows is left alone."""
    T, V = z.shape
    tok = tokens.cpu().numpy() if tokens is not None else None
    z64 = to_f64(z)
    want = orc.token_logprobs_backward(z64, tok, c, None if gl is None else to_f64(gl), None if gh is None else to_f64(gh))
    stats = torch.from_numpy(orc.token_logprobs(z64, None, c)["stats"].astype(np.float32)).cuda()
    if in_place:
        out = z
    elif out is None:
        out = torch.full_like(z, float("nan"))
    ql.qlora_token_logprobs_bwd(z, tokens, c, stats, gl, gh, out)
    got = to_f64(out)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = (z64 - z64.max(axis=1, keepdims=True)) * c
        lp = d - np.log(np.exp(d).sum(axis=1, keepdims=True))
        p = np.exp(lp)
        a = np.zeros((T, 1)) if gl is None else np.abs(to_f64(gl))[:, None]
        b = np.zeros((T, 1)) if gh is None else np.abs(to_f64(gh))[:, None]
        ent = -np.where(p > 0, p * lp, 0.0).sum(axis=1, keepdims=True)
        size = c * np.where(p > 0, p * (a + b * (np.abs(lp) + ent)), 0.0)
        rel = chain(V) + 4 * U * (16 + np.abs(np.where(p > 0, lp, 0.0)))
        if tok is not None:
            for t in range(T):
                if 0 <= tok[t] < V:
                    size[t, tok[t]] += c * a[t, 0]
        info = torch.finfo(z.dtype)
        bound = info.eps / 2 * np.abs(want) + rel * size + info.tiny * info.eps + 1e-37
        off = np.abs(got - want)
    fine = (off <= bound) | (np.isnan(got) & np.isnan(want))
    assert fine.all(), (float(np.nanmax(off)), np.argwhere(~fine)[:3])
    return out, want


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,V,ld,offset", [(1, 1, 1, 0), (1, 32000, 32000, 0), (5, 7, 9, 1), (33, 4097, 4097, 0), (6, 1000, 1003, 5), (3, 2048, 2112, 8), (400, 520, 520, 0)])
@pytest.mark.parametrize("terms", ["token", "entropy", "both"])
def test_gradient(T, V, ld, offset, dtype, terms):
    z, tokens = make(T, V, dtype, seed=T + V, ld=ld, offset=offset)
    gen = torch.Generator(device="cuda").manual_seed(1)
    gl = torch.randn(T, device="cuda", generator=gen) if terms != "entropy" else None
    gh = torch.randn(T, device="cuda", generator=gen) if terms != "token" else None
    if T > 3:
        tokens[1], tokens[2] = -1, V
    check_backward(z, tokens if terms != "entropy" else None, 0.9, gl, gh)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradient_in_place_and_into_other_rows(dtype):
    z, tokens = make(12, 1001, dtype, seed=31, ld=1010, offset=3)
    gl, gh = torch.randn(12, device="cuda"), torch.randn(12, device="cuda")
    buf = torch.full((12 * 1024 + 64,), 5.0, dtype=z.dtype, device="cuda")
    out = buf[2:2 + 12 * 1024].view(12, 1024)[:, :1001]              # rows that begin elsewhere than those of the logits
    other, _ = check_backward(z, tokens, 1.0, gl, gh, out=out)
    kept = other.clone()
    whole = buf.clone()
    whole[2:2 + 12 * 1024].view(12, 1024)[:, :1001] = 5.0
    assert (whole == 5.0).all()                                      # nothing written between the rows
    check_backward(z, tokens, 1.0, gl, gh, in_place=True)
    assert torch.equal(z, kept)


def test_gradient_beside_the_logits_in_one_buffer():
    V = 777
    buf = torch.full((50, 1600), 3.0, dtype=torch.bfloat16, device="cuda")
    z, out = buf[:, 8:8 + V], buf[:, 808:808 + V]
    z.copy_(torch.randn((50, V), device="cuda"))
    kept = z.clone()
    check_backward(z, torch.arange(50, dtype=torch.int32, device="cuda"), 1.0, torch.ones(50, device="cuda"), None, out=out)
    assert torch.equal(z, kept) and (buf[:, :8] == 3).all() and (buf[:, 785:808] == 3).all() and (buf[:, 1585:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_gradient_of_masked_and_broken_rows(dtype):
    """Masked entries have none; a row with nothing left, or without a gradient, is zeros whatever it holds; a broken one is NaN."""
    V = 900
    z, tokens = make(8, V, dtype, seed=37)
    z[0, 10:800] = float("-inf")
    z[1] = float("-inf")
    z[2] = torch.finfo(z.dtype).min
    z[3, 50:] = torch.finfo(z.dtype).min
    z[4, 3] = float("nan")                                           # no gradient: zeros
    z[5, 3] = float("nan")
    z[6, 3] = float("inf")
    tokens[0], tokens[4] = 5, -1
    gl, gh = torch.ones(8, device="cuda"), torch.full((8,), 0.5, device="cuda")
    gh[4] = 0.0
    out, want = check_backward(z, tokens, 1.0, gl, gh)
    assert (out[0, 10:800] == 0).all() and (out[1] == 0).all() and (out[4] == 0).all() and torch.isnan(out[5]).all() and torch.isnan(out[6]).all()


def test_gradient_against_differences():
    """Along a random unit direction d, for logits of spread 1: the difference quotient of the forward call over 2h has a truncation error
    below h^2 (third derivatives are below 6 along a unit direction) and a rounding error of 8 chain(V) (1 + 25) / 2h; h = 2^-5."""
    V, h = 64, 2.0 ** -5
    z, tokens = make(6, V, "fp32", seed=41, spread=1.0)
    d = torch.randn_like(z)
    d /= d.norm(dim=1, keepdim=True)
    gl, gh = torch.rand(6, device="cuda"), torch.rand(6, device="cuda")

    def total(x):
        out = forward(x.contiguous(), tokens, 1.0, 0)
        return to_f64(out["logprobs"]) * to_f64(gl) + to_f64(out["entropy"]) * to_f64(gh)
    stats = forward(z, tokens, 1.0, 0)["stats"]
    grad = torch.empty_like(z)
    ql.qlora_token_logprobs_bwd(z, tokens, 1.0, stats, gl, gh, grad)
    want = (total(z + h * d) - total(z - h * d)) / (2 * h)
    assert np.abs(to_f64((grad * d).sum(1)) - want).max() <= 2 * h * h + 8 * chain(V) * 26 / (2 * h)


def test_the_longest_row_and_very_many_short_ones():
    """2^24 logits; 200000 rows of 5.  The reference is the formula in 64 bits on the GPU (the oracle goes row by row)."""
    for T, V, k in ((1, 1 << 24, 5), (200000, 5, 3)):
        z, tokens = make(T, V, "fp16", seed=53)
        out = forward(z, tokens, 1.0, k)
        lp = torch.log_softmax(z.double(), 1)
        close(out["logprobs"], lp.gather(1, tokens.long()[:, None]).squeeze(1).cpu().numpy(), chain(V))
        close(out["entropy"], -(lp.exp() * lp).sum(1).cpu().numpy(), 25 * chain(V))
        order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(out["top_ids"].long(), order)
        close(out["top_logprobs"], lp.gather(1, order).cpu().numpy(), chain(V))
        grad = torch.empty_like(z)
        ql.qlora_token_logprobs_bwd(z, tokens, 1.0, out["stats"], torch.ones(T, device="cuda"), None, grad)
        want = -lp.exp()
        want.scatter_add_(1, tokens.long()[:, None], torch.ones_like(want[:, :1]))
        size = lp.exp().scatter_add(1, tokens.long()[:, None], torch.ones_like(want[:, :1]))
        bound = 2.0 ** -11 * want.abs() + (chain(V) + 4 * U * (16 + lp.abs())) * size + 2.0 ** -24
        assert ((grad.double() - want).abs() <= bound).all()


def test_long_offsets():
    """A row that begins beyond 2^31 elements."""
    rows, ld = 3, (1 << 30) + 8
    buf = torch.empty(2 * ld + 4000, dtype=torch.float16, device="cuda")
    z = torch.as_strided(buf, (rows, 4000), (ld, 1))
    z.copy_(torch.randn((rows, 4000), device="cuda"))
    tokens = torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda")
    check_forward(z, tokens, 1.0, 4)
    check_backward(z, tokens, 1.0, torch.ones(rows, device="cuda"), None, in_place=True)


def test_captured_and_replayed_on_other_logits():
    z, tokens = make(9, 5000, "bf16", seed=43)
    out = forward(z, tokens, 1.0, 4)
    grad = torch.empty_like(z)
    gl = torch.ones(9, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            ql.qlora_token_logprobs(z, tokens, 1.0, out["logprobs"], entropy=out["entropy"], top_ids=out["top_ids"], top_logprobs=out["top_logprobs"], stats=out["stats"])
            ql.qlora_token_logprobs_bwd(z, tokens, 1.0, out["stats"], gl, None, grad)
    for seed in (1, 2):
        z.copy_(make(9, 5000, "bf16", seed=seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        want = forward(z, tokens, 1.0, 4)
        for key in want:
            assert torch.equal(out[key], want[key]), key
        again = torch.empty_like(z)
        ql.qlora_token_logprobs_bwd(z, tokens, 1.0, want["stats"], gl, None, again)
        assert torch.equal(grad, again)


def test_two_streams_at_once():
    pairs = [make(40, 8000 + 8 * i, "bf16", seed=47 + i) for i in range(2)]
    want = [forward(z, t, 1.0, 10) for z, t in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, (z, t) in zip(streams, pairs):
            with torch.cuda.stream(s):
                got.append(forward(z, t, 1.0, 10))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(a[k], b[k]) for k in a)
