"""Log probabilities and their gradient where the temperature times the logits is large: rows masked altogether by a large negative number,
large logits, temperatures down to 2^-30 (needs a B200).  The reference is the formula in 64 bits.

Tolerances (u = 2^-24).  A row is summed either in base 2 relative to its maximum or from the differences to it; in both, d = c (z - max) carries a
relative error of 3u, exp(d) one of 3u |d| (at most 2u of the sum, |d| e^d < 0.4) + 2^-21, and a sum of V positive terms is formed along chains of at most
V / 256 + 64 additions here (V / 64 of up to 1000 logits, V / 128 of up to 7000, V / 256 of more).  So log s is off by at most S = (V / 256 + 64) u, a log probability by
S + 4u |log p|, the entropy log s - (sum e d) / s by S + (S + 8u) times the mean of |d|, which is H - log s <= log V < 11: 25 S covers
both.
Gradients, from the kernel's own statistics: p is off by S (log s) + S + 4u (16 + |log p|) relatively, H by 25 S, and the result is rounded once to its type (half a
step)."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# Rows and vocabularies that each way of sharing rows out takes: many very short rows, short ones, rows of up to 32 KB, few, some hundred, many.
WAYS = [(3000, 331, 5), (40, 1000, 0), (40, 1000, 5), (170, 7000, 5), (40, 20011, 0), (40, 20011, 5), (300, 20011, 0), (300, 40000, 5), (460, 12001, 5), (460, 20011, 5),
        (460, 40000, 0), (460, 40000, 5)]


def chain(V):
    return (V / 256 + 64) * U


def make(T, V, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn((T, V), device="cuda", generator=gen) * 3).to(DTYPES[dtype])
    return z, torch.randint(0, V, (T,), device="cuda", generator=gen).int(), gen


def check(z, tokens, c, k, gen):
    """The forward call, and the gradient from the statistics that it leaves."""
    T, V = z.shape
    c = torch.tensor(c, dtype=torch.float32).item()
    new = lambda *shape, dtype=torch.float32: torch.full(shape, -7, dtype=dtype, device="cuda")  # noqa: E731
    lp, ent, stats = new(T), new(T), new(T, 3)
    ids, top = (new(T, k, dtype=torch.int32), new(T, k)) if k else (None, None)
    ql.qlora_token_logprobs(z, tokens, c, lp, entropy=ent, top_ids=ids, top_logprobs=top, stats=stats)
    z64, at = z.double(), tokens.long()[:, None]
    m = z64.amax(1, keepdim=True)
    d = (z64 - m) * c
    e = d.exp()
    s = e.sum(1, keepdim=True)
    logs = s.log()
    H = logs - (e * d).sum(1, keepdim=True) / s
    logp = d - logs
    S = chain(V)
    agree(stats[:, 0], m[:, 0], 0.0, 0.0)
    agree(stats[:, 1], logs[:, 0], S, 4 * U)
    agree(ent, H[:, 0], 25 * S, 4 * U)
    assert torch.equal(ent, stats[:, 2])
    agree(lp, logp.gather(1, at)[:, 0], S, 4 * U)
    if k:
        order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids.long(), order)
        agree(top, logp.gather(1, order), S, 4 * U)
    gl, gh = (torch.randn(T, device="cuda", generator=gen) / c for _ in range(2))
    dz = torch.empty_like(z)
    ql.qlora_token_logprobs_bwd(z, tokens, c, stats, gl, gh, dz)
    p, a, b = logp.exp(), c * gl.double()[:, None], c * gh.double()[:, None]
    want = -p * (a + b * torch.where(p > 0, logp + H, 0.0))
    want.scatter_add_(1, at, a)
    size = p * (a.abs() + b.abs() * (torch.where(p > 0, logp.abs(), 0.0) + H + 25))
    off = size * (2 * S + 4 * U * (16 + torch.where(p > 0, logp.abs(), 0.0)))
    off.scatter_add_(1, at, 4 * U * a.abs())
    info = torch.finfo(z.dtype)
    off += info.eps / 2 * (want.abs() + off) + info.tiny * info.eps + 1e-37
    assert (((dz.double() - want).abs() <= off)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,k", WAYS)
def test_rows_masked_by_large_numbers_and_large_logits(T, V, k, dtype):
    """Rows of one large number, and ordinary logits of which all but one, all but two or half are masked by one, among ordinary rows."""
    z, tokens, gen = make(T, V, dtype, seed=T + V + k)
    row = iter(range(0, T, T // 40))
    for value in (-1e9, -1e10, -1e12, -1e20, -2.0 ** 80, 3e9, 1e12, 2.0 ** 60, 1e30):
        z[next(row)] = value
    for value in (-1e6, -1e9, -1e10, -1e20):
        for left in (1, 2, V // 2):
            t = next(row)
            z[t, left:] = value
            if left == 2:
                z[t, :2] = 12.0625
    t = next(row)
    z[t] = -1e10                                                   # two large numbers
    z[t, 3] = 1e10
    t = next(row)
    z[t] += 1e10                                                   # (in fp32 differences of 1024)
    tokens[::3] = 0
    check(z, tokens, 1.0, k, gen)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,V,k", WAYS)
@pytest.mark.parametrize("c", [1e5, 1e6, 1e8, 3e8, 1e9, 2.0 ** 30, 2.0 ** -30])
def test_temperatures_down_to_the_smallest(T, V, k, dtype, c):
    """Ordinary rows, one largest logit, two equal ones, all equal, masked in part and altogether by fp16's lowest value."""
    z, tokens, gen = make(T, V, dtype, seed=T + V + k)
    row = iter(range(0, T, T // 20))
    z[next(row), :3] = torch.tensor([33.4375, 1.0, -2.0], device="cuda").to(z.dtype)
    z[next(row), :2] = 32.0625
    for value in (20.3, -20.3, 0.0, -65504.0, 60000.0):
        z[next(row)] = value
    for left in (1, 2, V // 2):
        z[next(row), left:] = -65504.0
    t = next(row)
    z[t] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 15.0, -15.0).to(z.dtype)
    tokens[::3] = 0
    check(z, tokens, c, k, gen)


@pytest.mark.parametrize("power", [20, 23, 24, 25, 30, 31])
def test_around_the_border_between_the_two_ways_of_summing(power):
    """Maxima whose c log2(e) max lies around powers of two: the same tolerances on both sides."""
    V = 3001
    z, tokens, gen = make(64, V, "fp32", seed=power)
    kd = 1.4426950408889634
    top = 2.0 ** power / kd * (1 + torch.linspace(-1e-3, 1e-3, 32, device="cuda", dtype=torch.float64))
    level = torch.cat((top, -top))[:, None]
    step = 2.0 ** max(power - 23, 0)
    z.copy_((level.float() - step * torch.randint(0, 12, z.shape, device="cuda", generator=gen)))
    tokens[:] = torch.randint(0, V, (64,), device="cuda", generator=gen).int()
    check(z, tokens, 1.0, 7, gen)
