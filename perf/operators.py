"""The operators around the layer that a fine-tuning program has next to it, as measurable cases.

Kinds of work:
  logprobs      log probabilities of given tokens over [tokens, vocabulary] logits, the entropy of each row and its most
                likely alternatives: evaluation (perplexity), generation, a teacher's targets to be kept
  logprobs_bwd  their gradient with respect to the logits
  adamw         one AdamW step over every LoRA pair of a model, with states in 32 or in 8 bits, most often behind the
                clipping of the gradients' global norm

Where `own` is false every operator is computed in its plain form, with elementary torch operations.

Logits are N(0, 3) with a few tokens of each row raised far above the rest, as a language model's are; LoRA gradients are
normal with a size of their own for each tensor, and the moments are those of such gradients.
"""
import itertools
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BLOCK = 256                  # elements that share one scale where states are held in 8 bits
E4M3_MAX = 448.0
E4M3_TINY = 2.0 ** -9        # the smallest positive e4m3 value
TINY_SCALE = 2.0 ** -100     # a block with nothing above it is held as zeros
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 3e-4


def logprobs(name=None, **kw):
    case = dict(name=name, kind="logprobs", dtype="bf16", T=2048, V=32000, ld=32000, k=0, temperature=1.0, masked=0.0)
    case.update(kw)
    return {k: v for k, v in case.items() if v is not None}


def backward(name=None, **kw):
    case = dict(name=name, kind="logprobs_bwd", dtype="bf16", T=2048, V=32000, ld=32000, temperature=1.0, entropy=True, padded=0.0)
    case.update(kw)
    return {k: v for k, v in case.items() if v is not None}


def adamw(name=None, **kw):
    case = dict(name=name, kind="adamw", bits=32, layers=32, sites="qkvogud", hidden=4096, inner=11008, r=8, param="bf16", grad="fp32",
                master=False, clip=True, device_step=False)
    case.update(kw)
    return {k: v for k, v in case.items() if v is not None}


def listed():
    return [
        # Generating one token: its log probability and twenty alternatives.
        logprobs("token_top20", T=1, k=20),
        # Sixteen sequences in step, half of the vocabulary ruled out, a vocabulary padded to a multiple of 64, sampling temperature.
        logprobs("tokens_16_masked_top5", T=16, ld=32064, k=5, temperature=0.7, masked=0.5),
        # Perplexity of a text of 2048 tokens.
        logprobs("perplexity_2048", T=2048),
        # The targets of a teacher, kept as the 32 most likely tokens of each place.
        logprobs("teacher_top32_2048", dtype="fp16", T=2048, k=32),
        # A vocabulary of an odd size, rows that start anywhere.
        logprobs("odd_vocabulary_top8", dtype="fp32", T=1031, V=50021, ld=50021, k=8, temperature=1.3),
        # A long batch over a large vocabulary.
        logprobs("large_4096_128000_top20", T=4096, V=128000, ld=128000, k=20),
        # Policy gradient with an entropy term, 4 x 512 tokens.
        backward("gradient_2048", T=2048),
        # Cross-entropy alone over fp32 logits of an odd vocabulary, a third of the places padding.
        backward("gradient_odd_padded", dtype="fp32", T=777, V=50021, ld=50021, entropy=False, padded=0.33),
        # The two adapter matrices of one projection: launches and latency are all there is.
        adamw("adamw_one_pair", layers=1, sites="q"),
        # The paper's fine-tuning setting, rank 8 on q and v of 32 layers, 8-bit states.
        adamw("adamw8_qv_r8", bits=8, sites="qv"),
        # Rank 32 on all seven projections of 32 layers, 8-bit states.
        adamw("adamw8_all_r32", bits=8, r=32),
        # Rank 64 on all seven projections, 32-bit states and fp32 master weights.
        adamw("adamw_all_r64_master", r=64, master=True),
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, uniform in its logarithm."""
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choices(("logprobs", "logprobs_bwd", "adamw"), (0.4, 0.2, 0.4))[0]
    if kind == "adamw":
        hidden = _spread(rng, 256, 4096)
        bits = rng.choice((8, 32))
        return adamw(bits=bits, layers=rng.choice((1, 2, 16, 32)), sites=rng.choice(("q", "qv", "qkvo", "qkvogud")), hidden=hidden,
                     inner=_spread(rng, hidden, 11008), r=rng.choice((4, 8, 16, 24, 32, 64)), param=rng.choice(("bf16", "bf16", "fp16")),
                     grad=rng.choice(("fp32", "fp32", "bf16")), master=rng.random() < 0.4, clip=rng.random() < 0.6, device_step=rng.random() < 0.3)
    V = _spread(rng, 2000, 130000)
    T = _spread(rng, 1, 8192)
    while T * V > 4096 * 128000 // 2:
        T = T // 2 + 1
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    ld = V + rng.choice((0, 0, 1, 64 - V % 64))
    temperature = rng.choice((1.0, 1.0, 0.6, 1.5))
    if kind == "logprobs_bwd":
        return backward(dtype=dtype, T=T, V=V, ld=ld, temperature=temperature, entropy=rng.random() < 0.5, padded=rng.choice((0.0, 0.25)))
    return logprobs(dtype=dtype, T=T, V=V, ld=ld, k=rng.choice((0, 1, 5, 20, 32, 64)), temperature=temperature, masked=rng.choice((0.0, 0.0, 0.5)))


# ---------------------------------------------------------------------------------------------- inputs

def _logits(case, gen):
    T, V, dev = case["T"], case["V"], gen.device
    z = torch.empty((T, case["ld"]), dtype=DTYPES[case["dtype"]], device=dev).normal_(0.0, 3.0, generator=gen)
    raised = torch.randint(0, V, (T, 8), device=dev, generator=gen)
    lift = 8.0 + 6.0 * torch.rand((T, 8), device=dev, generator=gen)
    z.scatter_(1, raised, lift.to(z.dtype))
    if case.get("masked", 0.0) > 0.0:
        z.masked_fill_(torch.rand((T, case["ld"]), device=dev, generator=gen) < case["masked"], float("-inf"))
        z[:, 0] = 1.0                                              # (every row keeps one)
    tokens = raised[:, 0].to(torch.int32).contiguous()
    if case.get("padded", 0.0) > 0.0:
        tokens[torch.rand((T,), device=dev, generator=gen) < case["padded"]] = -1
    return z[:, :V], tokens


def _shapes(case):
    h, i, r = case["hidden"], case["inner"], case["r"]
    size = {"q": (h, h), "k": (h, h), "v": (h, h), "o": (h, h), "g": (h, i), "u": (h, i), "d": (i, h)}
    return [n * r for _ in range(case["layers"]) for s in case["sites"] for n in size[s]]


def _lay_out(case):
    """Where the tensors of the model lie in flat buffers: each begins at a multiple of 256 elements."""
    sizes = _shapes(case)
    ends = list(itertools.accumulate(-(-n // BLOCK) * BLOCK for n in sizes))
    return sizes, [0] + ends[:-1], ends[-1]


def _scaled(x):
    """Blocks of 256 values on the range of e4m3 numbers, not rounded, and the scale of each block."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1)
    held = top > TINY_SCALE
    scale = torch.where(held, top * (1.0 / E4M3_MAX), torch.zeros_like(top))
    code = x * torch.where(held, E4M3_MAX / top, torch.zeros_like(top))[:, None]
    return code.clamp(-E4M3_MAX, E4M3_MAX), scale


def _dithered(x, dither):
    """To an e4m3 number beside x, upward (in size) with a chance that is x's share of the step: `dither` is in [0, 2^20)."""
    a = x.abs()
    low = a < 2.0 ** -6                                            # (below, the steps are as large as in the first binade)
    y = torch.where(low, a + 2.0 ** -6, a)
    y = ((y.view(torch.int32) + dither.view_as(y)) & ~0xFFFFF).view(torch.float32)
    return torch.where(low, y - 2.0 ** -6, y).clamp_max(E4M3_MAX).copysign(x)


def _dithers(s, total):
    """Two numbers in [0, 2^20) for each element, from its place in its tensor and the number of the step."""
    place = torch.arange(total, device=s["starts"].device) - s["starts"].repeat_interleave(s["lengths"], output_size=total)
    x = (place * 0x9E3779B1 + s["step"] * 0x7F4A7C15) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
    x = ((x ^ (x >> 13)) * 0x297A2D39) & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return (x >> 12).int(), (((x * 0x9E3779B1) & 0xFFFFFFFF) >> 12).int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev, state = gen.device, dict(case=case)
    if case["kind"] == "adamw":
        sizes, starts, total = _lay_out(case)
        real = torch.zeros(total, dtype=torch.float32, device=dev)
        sigma = torch.zeros(total, dtype=torch.float32, device=dev)
        size_of = (torch.randn(len(sizes), device=dev, generator=gen) - 7.0).exp()
        for j, (n, a) in enumerate(zip(sizes, starts)):
            real[a:a + n] = 1.0
            sigma[a:a + n] = size_of[j]
        randn = lambda: torch.randn(total, device=dev, generator=gen)  # noqa: E731
        p = 0.02 * randn() * real
        state["param"] = p.to(DTYPES[case["param"]])
        if case["master"]:
            state["master"] = p
        state["grad"] = (sigma * randn()).to(DTYPES[case["grad"]])
        m, u = 0.3 * sigma * randn(), sigma * (0.3 + 0.7 * randn().abs())
        if case["bits"] == 8:
            code, state["m_scale"] = _scaled(m)
            state["m"] = code.to(torch.float8_e4m3fn).view(-1)
            code, state["v_scale"] = _scaled(u)                    # (held as its root)
            state["v"] = code.to(torch.float8_e4m3fn).view(-1)
            state["starts"] = torch.tensor(starts, device=dev)
            state["lengths"] = torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], device=dev)
        else:
            state["m"], state["v"] = m, u * u
        if case["clip"]:
            state["norm"] = torch.zeros(2, dtype=torch.float32, device=dev)
        state["lr"], state["step"] = LR, 100
        if case["device_step"]:                                    # a captured step, whose rate and number change between replays
            state["lr"] = torch.tensor([LR], dtype=torch.float32, device=dev)
            state["step"] = torch.tensor([100], dtype=torch.int32, device=dev)
        if own:
            import paper_2306_08162_b200 as ql

            def views(key, div=1):
                if key not in state:
                    return None
                return [state[key][a // div:a // div + -(-n // div)] for n, a in zip(sizes, starts)]
            state["workspace"] = torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=dev)
            state["desc"] = ql.adamw_desc(views("param"), views("grad"), views("m"), views("v"), master=views("master"),
                                          m_scale=views("m_scale", BLOCK), v_scale=views("v_scale", BLOCK),
                                          beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY)
        return state
    state["logits"], state["tokens"] = _logits(case, gen)
    T, V = case["T"], case["V"]
    if case["kind"] == "logprobs":
        state["logprobs"], state["entropy"] = (torch.empty(T, dtype=torch.float32, device=dev) for _ in range(2))
        state["stats"] = torch.empty((T, 3), dtype=torch.float32, device=dev)
        state["top_ids"] = torch.empty((T, case["k"]), dtype=torch.int32, device=dev) if case["k"] else None
        state["top_logprobs"] = torch.empty((T, case["k"]), dtype=torch.float32, device=dev) if case["k"] else None
        return state
    # what the forward pass has left for the backward pass: row maximum, logarithm of the sum, entropy
    stats = []
    for rows in state["logits"].split(256):
        d = rows.double()
        m = d.amax(1, keepdim=True)
        d = (d - m) / case["temperature"]
        logs = d.exp().sum(1, keepdim=True).log()
        stats.append(torch.cat((m, logs, -((d - logs).exp() * (d - logs)).sum(1, keepdim=True)), 1).float())
    state["stats"] = torch.cat(stats)
    state["d_logprobs"] = -torch.rand(T, device=dev, generator=gen) / T
    state["d_entropy"] = torch.full((T,), -0.01 / T, device=dev) if case["entropy"] else None
    state["dlogits"] = torch.zeros((T, case["ld"]), dtype=DTYPES[case["dtype"]], device=dev)[:, :V]
    return state


# ---------------------------------------------------------------------------------------------- one pass

def _plain_logprobs(s):
    case = s["case"]
    z = s["logits"].float()
    m = z.amax(1, keepdim=True)
    d = (z - m) * (1.0 / case["temperature"])
    e = d.exp()
    total = e.sum(1, keepdim=True)
    logs = total.log()
    mean = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, keepdim=True) / total
    entropy = (logs - mean).squeeze(1)
    token = s["tokens"].long()
    known = (token >= 0) & (token < case["V"])
    at = token.clamp(0, case["V"] - 1)[:, None]
    lp = torch.where(known, (d.gather(1, at) - logs).squeeze(1), torch.zeros_like(entropy))
    out = dict(logprobs=lp, entropy=entropy, stats=torch.cat((m, logs, entropy[:, None]), 1))
    if case["k"]:
        # one number for (logit, place): equal logits are in the order of their places
        del e
        bits = (z + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        key = key * (1 << 32) + (case["V"] - 1 - torch.arange(case["V"], device=z.device))
        ids = case["V"] - 1 - (key.topk(case["k"], dim=1).values & 0xFFFFFFFF)
        out["top_ids"], out["top_logprobs"] = ids.int(), d.gather(1, ids) - logs
    return out


def _plain_backward(s):
    case = s["case"]
    c = 1.0 / case["temperature"]
    m, logs, entropy = s["stats"].split(1, 1)
    lp = (s["logits"].float() - m) * c - logs
    p = lp.exp()
    token = s["tokens"].long()
    known = (token >= 0) & (token < case["V"])
    gl = torch.where(known, s["d_logprobs"], torch.zeros_like(s["d_logprobs"]))[:, None]
    if s["d_entropy"] is None:
        dz = p * (-c * gl)
    else:
        w = torch.where(p > 0, lp + entropy, torch.zeros_like(p))
        dz = -c * p * (gl + s["d_entropy"][:, None] * w)
    dz.scatter_add_(1, token.clamp(0, case["V"] - 1)[:, None], c * gl)
    return dz.to(DTYPES[case["dtype"]])


def _plain_adamw(s):
    case = s["case"]
    g = s["grad"].float()
    out = {}
    if case["clip"]:
        norm = s["grad"].double().square().sum().sqrt().float()
        factor = torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm))
        s["norm"].copy_(torch.stack((norm, factor)))
        out["norm"] = s["norm"]
        g = g * factor
    lr, t = s["lr"], s["step"]
    if case["device_step"]:
        t = t.double()
        c1, c2 = (1.0 - BETA1 ** t).float(), (1.0 - BETA2 ** t).float()
    else:
        c1, c2 = 1.0 - BETA1 ** t, 1.0 - BETA2 ** t
    if case["bits"] == 8:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        u = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * (u * u) + (1.0 - BETA2) * (g * g)
    else:
        m = s["m"].mul_(BETA1).add_((1.0 - BETA1) * g)
        v = s["v"].mul_(BETA2).add_((1.0 - BETA2) * (g * g))
    p = s["master"] if case["master"] else s["param"].float()
    p = p * (1.0 - lr * DECAY) - lr * ((m / c1) / ((v / c2).sqrt() + EPS))
    if case["master"]:
        out["master"] = s["master"].copy_(p)
    out["param"] = s["param"].copy_(p)
    if case["bits"] == 8:
        dither_m, dither_u = _dithers(s, m.numel())
        code, scale = _scaled(m)
        s["m"].view(-1, BLOCK).copy_(_dithered(code, dither_m))
        s["m_scale"].copy_(scale)
        code, scale = _scaled(v.sqrt())
        rounded = _dithered(code, dither_u)                        # what is above zero stays above zero
        s["v"].view(-1, BLOCK).copy_(torch.where(code > 0, rounded.clamp_min(E4M3_TINY), rounded))
        s["v_scale"].copy_(scale)
        out["m_scale"], out["v_scale"] = s["m_scale"], s["v_scale"]
    out["m"], out["v"] = s["m"], s["v"]
    return out


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"logprobs": _plain_logprobs, "logprobs_bwd": _plain_backward, "adamw": _plain_adamw}[case["kind"]](s)
    import paper_2306_08162_b200 as ql
    if case["kind"] == "logprobs":
        ql.qlora_token_logprobs(s["logits"], s["tokens"], 1.0 / case["temperature"], s["logprobs"], entropy=s["entropy"], top_ids=s["top_ids"],
                                top_logprobs=s["top_logprobs"], stats=s["stats"])
        names = ("logprobs", "entropy", "stats") + (("top_ids", "top_logprobs") if case["k"] else ())
        return {k: s[k] for k in names}
    if case["kind"] == "logprobs_bwd":
        ql.qlora_token_logprobs_bwd(s["logits"], s["tokens"], 1.0 / case["temperature"], s["stats"], s["d_logprobs"], s["d_entropy"], s["dlogits"])
        return s["dlogits"]
    if case["clip"]:
        ql.qlora_grad_norm(s["desc"], 1.0, 1.0, s["norm"], s["workspace"])
    ql.qlora_adamw(s["desc"], s["lr"], s["step"], s["norm"] if case["clip"] else None)
    return {k: s[k] for k in ("norm", "master", "param", "m_scale", "v_scale", "m", "v") if k in s}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "adamw":
        n = sum(_shapes(case))
        p, g = DTYPES[case["param"]].itemsize, DTYPES[case["grad"]].itemsize
        state = 2 * (2 * (1 + 4 / BLOCK)) if case["bits"] == 8 else 16
        weights = (8 + p) if case["master"] else 2 * p             # (a master weight is what is read; the parameter is written beside it)
        return {"bytes": n * (g + state + weights), "flops": 14 * n}
    T, V, size = case["T"], case["V"], DTYPES[case["dtype"]].itemsize
    if case["kind"] == "logprobs":
        return {"bytes": T * (V * size + 4 + 8 + 12 + 8 * case["k"]), "flops": 6 * T * V}
    with_gradient = 1.0 if case["entropy"] else 1.0 - case["padded"]
    return {"bytes": T * (V * size * (1 + with_gradient) + 20), "flops": 6 * T * V * with_gradient}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _row_blocks(case):
    rows = max(1, (1 << 26) // case["V"])
    return [(a, min(a + rows, case["T"])) for a in range(0, case["T"], rows)]


def _exact_rows(case, s, a, b):
    z = s["logits"][a:b].double() / case["temperature"]
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    entropy = torch.special.entr(lp.exp()).sum(1)
    token = s["tokens"][a:b].long()
    known = (token >= 0) & (token < case["V"])
    chosen = torch.where(known, lp[torch.arange(b - a, device=z.device), token % case["V"]], torch.zeros_like(lse))
    top = z.max(1).values
    out = dict(logprobs=chosen, entropy=entropy, stats=torch.stack((top * case["temperature"], lse - top, entropy), 1))
    if case["k"]:
        out["top_logprobs"] = lp.sort(1, descending=True).values[:, :case["k"]].contiguous()
    return out


def _exact_gradient_rows(case, s, a, b):
    z = (s["logits"][a:b].double() / case["temperature"]).requires_grad_(True)
    lp = torch.log_softmax(z, 1)
    token = s["tokens"][a:b].long()
    known = (token >= 0) & (token < case["V"])
    total = (lp[torch.arange(b - a, device=z.device), token % case["V"]] * s["d_logprobs"][a:b].double())[known].sum()
    if s["d_entropy"] is not None:
        total = total - ((lp.exp() * lp).sum(1) * s["d_entropy"][a:b].double()).sum()
    return torch.autograd.grad(total, z)[0] / case["temperature"]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "logprobs_bwd":
        return torch.cat([_exact_gradient_rows(case, s, a, b) for a, b in _row_blocks(case)])
    if case["kind"] == "logprobs":
        parts = [_exact_rows(case, s, a, b) for a, b in _row_blocks(case)]
        out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
        if case["k"]:
            out["top_ids"] = None
        return out
    sizes, starts, total = _lay_out(case)
    blank = lambda n=total: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    out = dict(param=blank(), m=blank(), v=blank())
    eight = case["bits"] == 8
    if eight:
        out["m_scale"], out["v_scale"] = blank(total // BLOCK), blank(total // BLOCK)
    f = 1.0
    if case["clip"]:
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(s["grad"][a:a + n].double())) ** 2 for n, a in zip(sizes, starts)))
        f = 1.0 / max(norm, 1.0)
        out["norm"] = torch.tensor([norm, f], dtype=torch.float64, device="cuda")
    for n, a in zip(sizes, starts):
        end = a + -(-n // BLOCK) * BLOCK
        g = f * s["grad"][a:end].double()
        m, v = s["m"][a:end].to(torch.float64), s["v"][a:end].to(torch.float64)
        if eight:
            m = m * s["m_scale"][a // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK)
            v = (v * s["v_scale"][a // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK)) ** 2
        m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g ** 2 - v)
        p = (s["master"] if case["master"] else s["param"])[a:end].double()
        out["param"][a:end] = p - LR * (DECAY * p + m / (1 - BETA1 ** 100) / (torch.sqrt(v / (1 - BETA2 ** 100)) + EPS))
        if eight:
            for key, x in (("m", m), ("v", v.sqrt())):
                scale = x.abs().view(-1, BLOCK).max(1).values / E4M3_MAX
                out[key + "_scale"][a // BLOCK:end // BLOCK] = scale
                out[key][a:end] = x / scale.clamp_min(1e-300).repeat_interleave(BLOCK)      # (what the codes round)
        else:
            out["m"][a:end], out["v"][a:end] = m, v
    if case["master"]:
        out["master"] = out["param"]
    return out
