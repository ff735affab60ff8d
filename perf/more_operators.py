"""A step of several adapters on one frozen base, as measurable cases: the low-rank adapters of many requests beside a shared
projection, and the cross entropy of the model's head taken from the hidden states.

Kinds of work:
  adapters       Y = Y_base + s_a (X A_a^T) B_a^T, where every token has an adapter a of its own or none: generating a token for
                 many requests, prompts of some requests beside single tokens of others, the forward pass of a training batch
  adapters_back  the same backward: dX = dX_base + s_a (dY B_a) A_a
  adapters_grad  the gradients of every adapter's pair: dA_a = s_a G^T X, dB_a = s_a dY^T H over the tokens of a
  head_loss      cross entropy of given labels under softmax(hidden W^T), where the logits are not kept: alone (scoring a text),
                 or with its gradient with respect to the hidden states (training)

Where `own` is false every operator is computed in its plain form, with elementary torch operations.

Adapters are A ~ U(-1/sqrt(K), 1/sqrt(K)) and B ~ N(0, 0.05), as after some training; activations are N(0, 1).  The head is
N(0, 0.02); hidden states lie nearer to their label's row, some so near that the label has almost all of the probability.
"""
import math

import torch

own = False


def adapters(name=None, **kw):
    """`prompts` requests of random lengths and `singles` of one token, M tokens in all, take the L adapters in turn; with `bare`
    every seventh request has none."""
    case = dict(name=name, kind="adapters", M=2048, K=4096, N=4096, r=16, L=8, prompts=8, singles=0, bare=False)
    case.update(kw)
    return {k: v for k, v in case.items() if v is not None}


def head(name=None, **kw):
    case = dict(name=name, kind="head_loss", T=2048, V=32000, D=4096, gradient=True, padded=0.0)
    case.update(kw)
    return {k: v for k, v in case.items() if v is not None}


def listed():
    return [
        # Generating one token for one request: launches and latency are all there is.
        adapters("decode_1", M=1, prompts=0, singles=1),
        # Generating a token for 64 requests with adapters of their own, MLP up projection; some requests without one.
        adapters("decode_64", M=64, N=11008, L=96, prompts=0, singles=64, bare=True),
        # A serving step: a few prompts beside 48 requests in generation.
        adapters("mixed_1911", M=1911, r=32, L=24, prompts=5, singles=48, bare=True),
        # Training eight adapters on 8 x 512 tokens, MLP up projection: forward ...
        adapters("train_4096", M=4096, N=11008, L=8, prompts=8),
        # ... and the gradient with respect to the projection's input.
        adapters("back_4096", kind="adapters_back", M=4096, N=11008, r=8, L=8, prompts=8),
        # The adapters' gradients of such a batch on an attention projection.
        adapters("grad_4096", kind="adapters_grad", M=4096, L=8, prompts=8),
        # Ragged, an odd rank, some tokens without an adapter, one adapter's sequences in several places.
        adapters("grad_ragged_1531", kind="adapters_grad", M=1531, K=11008, r=24, L=5, prompts=13, bare=True),
        # Scoring the last tokens of 16 candidates.
        head("score_16", T=16, gradient=False),
        # Scoring a text of 2048 tokens.
        head("score_2048", gradient=False),
        # Fine-tuning, 4 x 512 tokens.
        head("loss_2048"),
        # A vocabulary of an odd size, a third of the places padding.
        head("loss_odd_777", T=777, V=50021, D=2568, padded=0.33),
        # A long batch over a large vocabulary.
        head("loss_8192_128000", T=8192, V=128000),
    ]


def _spread(rng, lo, hi, multiple=1):
    """A size between lo and hi, uniform in its logarithm, a multiple of `multiple`."""
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple)) * multiple)


def draw(rng):
    kind = rng.choices(("adapters", "adapters_back", "adapters_grad", "head_loss"), (0.3, 0.15, 0.2, 0.35))[0]
    if kind == "head_loss":
        T, V, D = _spread(rng, 1, 8192), _spread(rng, 2000, 130000), _spread(rng, 512, 4096, 8)
        while T * V * D > 8192 * 128000 * 4096 // 4:
            T = T // 2 + 1
        return head(T=T, V=V, D=D, gradient=rng.random() < 0.6, padded=rng.choice((0.0, 0.25)))
    K, N, r, L = _spread(rng, 512, 11008, 32), _spread(rng, 512, 11008, 8), rng.choice((8, 8, 16, 16, 24, 32, 64)), _spread(rng, 1, 64)
    if kind == "adapters" and rng.random() < 0.4:                  # generation
        M = _spread(rng, 1, 256)
        return adapters(M=M, K=K, N=N, r=r, L=L, prompts=0, singles=M, bare=rng.random() < 0.5)
    M = _spread(rng, 64, 8192)
    singles = rng.choice((0, 0, 1, 16, 40)) if kind == "adapters" else 0
    return adapters(kind=kind, M=M, K=K, N=N, r=r, L=L, prompts=_spread(rng, 1, 16), singles=singles, bare=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs

def _requests(case):
    """How many requests there are, and for each the adapter's number before shuffling, or -1."""
    n = case["prompts"] + case["singles"]
    return n, [-1 if case["bare"] and i % 7 == 3 else i % case["L"] for i in range(n)]


def _adapter_of(case, gen):
    """The adapter of each token: whole requests in a row, prompts cut at random places."""
    n, order = _requests(case)
    dev, prompts, long = gen.device, case["prompts"], case["M"] - case["singles"]
    first = torch.tensor(order, device=dev)
    shuffled = torch.randperm(case["L"], device=dev, generator=gen)
    adapter = torch.where(first >= 0, shuffled[first.clamp_min(0)], first)
    cuts = torch.randint(0, long + 1, (max(prompts - 1, 0),), device=dev, generator=gen).sort().values
    place = torch.arange(case["M"], device=dev)
    request = torch.searchsorted(cuts, place.clamp_max(max(long - 1, 0)), right=True) if prompts else torch.zeros_like(place)
    request = torch.where(place >= long, prompts + place - long, request)
    return adapter[request].to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev, s = gen.device, dict(case=case)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(0.0, std, generator=gen)

    if case["kind"] == "head_loss":
        T, V, D = case["T"], case["V"], case["D"]
        s["head"] = normal(V, D, std=0.02)
        label = torch.randint(0, V, (T,), device=dev, generator=gen)
        near = 12.0 * torch.rand((T, 1), device=dev, generator=gen) * (4096.0 / D) ** 0.5
        s["hidden"] = (2.0 * torch.randn((T, D), device=dev, generator=gen) + near * s["head"][label].float()).bfloat16()
        label[torch.rand((T,), device=dev, generator=gen) < case["padded"]] = -1
        s["labels"] = label.to(torch.int32)
        s["loss"] = torch.empty(T, dtype=torch.float32, device=dev)
        if case["gradient"]:
            s["d_loss"] = torch.full((T,), 1.0 / T, dtype=torch.float32, device=dev)
            s["d_hidden"] = torch.empty_like(s["hidden"])
        if own:
            import paper_2306_08162_b200 as ql
            s["workspace"] = torch.empty(ql.qlora_head_loss_workspace_bytes(T, V, D, case["gradient"]), dtype=torch.uint8, device=dev)
        return s
    M, K, N, r, L = (case[k] for k in ("M", "K", "N", "r", "L"))
    s["adapter_of"] = _adapter_of(case, gen)
    s["A"] = torch.empty((L, r, K), dtype=torch.bfloat16, device=dev).uniform_(-1 / math.sqrt(K), 1 / math.sqrt(K), generator=gen)
    s["B"] = normal(L, N, r, std=0.05)
    s["scales"] = 2.0 + 0.5 * torch.rand((L,), device=dev, generator=gen)
    known = (s["adapter_of"] >= 0).float()[:, None]
    if case["kind"] == "adapters":
        s["X"], s["base"] = normal(M, K), normal(M, N)
        s["out"], s["low"] = torch.empty_like(s["base"]), None
        if case["singles"] == 0:                                   # a training step keeps H
            s["low"] = torch.empty((M, r), dtype=torch.float32, device=dev)
    elif case["kind"] == "adapters_back":
        s["dY"], s["base"] = normal(M, N), normal(M, K)
        s["out"], s["low"] = torch.empty_like(s["base"]), torch.empty((M, r), dtype=torch.float32, device=dev)
    else:
        s["X"], s["dY"] = normal(M, K), normal(M, N)
        s["H"] = 0.6 * torch.randn((M, r), device=dev, generator=gen) * known
        s["G"] = 0.05 * math.sqrt(N) * torch.randn((M, r), device=dev, generator=gen) * known
        s["dA"] = torch.empty((L, r, K), dtype=torch.float32, device=dev)
        s["dB"] = torch.empty((L, N, r), dtype=torch.float32, device=dev)
    if own:
        import paper_2306_08162_b200 as ql
        s["desc"] = ql.adapters_desc(K, N, r, L)
        s["workspace"] = torch.empty(ql.qlora_adapters_workspace_bytes(s["desc"], M), dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def _chosen(s):
    """Ones where a token has an adapter: fp32 [M, L, 1]."""
    places = torch.arange(s["case"]["L"], device=s["adapter_of"].device)
    return (s["adapter_of"][:, None] == places).float()[:, :, None]


def _plain_adapters(s, x, down, up):
    """x [M, T], down [L r, T], up [L r, C]: every token against all adapters, its own kept."""
    case = s["case"]
    M, L, r = case["M"], case["L"], case["r"]
    low = (x.float() @ down.t()).view(M, L, r) * _chosen(s)
    out = s["base"].float() + (low * s["scales"][:, None]).view(M, L * r) @ up
    return (out.to(torch.bfloat16),) if s["low"] is None else (out.to(torch.bfloat16), low.sum(1))


def _plain_gradients(s):
    case = s["case"]
    M, K, N, r, L = (case[k] for k in ("M", "K", "N", "r", "L"))
    mine = _chosen(s) * s["scales"][:, None]
    dA = (s["G"][:, None] * mine).view(M, L * r).t() @ s["X"].float()
    dB = (s["H"][:, None] * mine).view(M, L * r).t() @ s["dY"].float()
    return dA.view(L, r, K), dB.view(L, r, N).transpose(1, 2).contiguous()


def _plain_head(s):
    case = s["case"]
    w = s["head"].float()
    z = s["hidden"].float() @ w.t()
    z -= z.amax(1, keepdim=True)
    label = s["labels"].long()
    known = (label >= 0) & (label < case["V"])
    at = label.clamp(0, case["V"] - 1)[:, None]
    mine = z.gather(1, at).squeeze(1)
    z.exp_()
    total = z.sum(1)
    loss = torch.where(known, total.log() - mine, torch.zeros_like(mine))
    if not case["gradient"]:
        return (loss,)
    d = torch.where(known, s["d_loss"], torch.zeros_like(mine))
    z *= (d / total)[:, None]
    z.scatter_add_(1, at, -d[:, None])
    return loss, (z @ w).to(torch.bfloat16)


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "head_loss":
            return _plain_head(s)
        if kind == "adapters_grad":
            return _plain_gradients(s)
        A, B = s["A"].float().flatten(0, 1), s["B"].float().transpose(1, 2).flatten(0, 1)
        return _plain_adapters(s, s["X"], A, B) if kind == "adapters" else _plain_adapters(s, s["dY"], B, A)
    import paper_2306_08162_b200 as ql
    if kind == "head_loss":
        ql.qlora_head_loss(s["hidden"], s["head"], s["labels"], s["loss"], s["workspace"], d_loss=s.get("d_loss"), d_hidden=s.get("d_hidden"))
        return (s["loss"], s["d_hidden"]) if case["gradient"] else (s["loss"],)
    if kind == "adapters_grad":
        ql.qlora_adapters_bwd_lora(s["desc"], case["M"], s["X"], s["dY"], s["adapter_of"], s["A"], s["B"], s["scales"], s["H"], s["G"], s["dA"], s["dB"], 0,
                                   s["workspace"])
        return s["dA"], s["dB"]
    if kind == "adapters":
        ql.qlora_adapters_fwd(s["desc"], case["M"], s["X"], s["adapter_of"], s["A"], s["B"], s["scales"], s["base"], s["out"], s["low"], s["workspace"])
    else:
        ql.qlora_adapters_bwd_input(s["desc"], case["M"], s["dY"], s["adapter_of"], s["A"], s["B"], s["scales"], s["base"], s["out"], s["low"], s["workspace"])
    return (s["out"],) if s["low"] is None else (s["out"], s["low"])


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "head_loss":
        T, V, D = case["T"], case["V"], case["D"]
        real = 1.0 - case["padded"]                                # (a padded token has neither a loss nor a gradient)
        moved = V * D * 2 + T * (real * D * 2 + 8) + (T * (D * 2 + 4) if case["gradient"] else 0)
        return {"bytes": moved, "flops": (4 if case["gradient"] else 2) * real * T * V * D}
    M, K, N, r = (case[k] for k in ("M", "K", "N", "r"))
    n, order = _requests(case)
    prompts, long = case["prompts"], M - case["singles"]
    used, served = len({a for a in order if a >= 0}), sum(a >= 0 for a in order[prompts:])
    share = (served + (long * sum(a >= 0 for a in order[:prompts]) / prompts if prompts else 0)) / M      # of the tokens, on average
    if case["kind"] == "adapters_grad":
        return {"bytes": share * M * ((K + N) * 2 + 8 * r) + 4 * M + case["L"] * r * (K + N) * 4, "flops": share * 2 * M * r * (K + N)}
    into, out = (K, N) if case["kind"] == "adapters" else (N, K)
    low = 4 * r * M if case["kind"] == "adapters_back" or case["singles"] == 0 else 0
    return {"bytes": 2 * M * (share * into + 2 * out) + 4 * M + used * r * (K + N) * 2 + low, "flops": share * 2 * M * r * (K + N)}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_head(case, s):
    T, V = case["T"], case["V"]
    w = s["head"].double()
    losses, grads = [], []
    rows = max(1, (1 << 27) // V)
    for a in range(0, T, rows):
        h = s["hidden"][a:a + rows].double()
        lp = torch.log_softmax(torch.einsum("td,vd->tv", h, w), 1)
        label = s["labels"][a:a + rows].long()
        known = (label >= 0) & (label < V)
        here = torch.arange(len(label), device=lp.device)
        losses.append(torch.where(known, -lp[here, label % V], 0.0))
        if case["gradient"]:
            p = lp.exp_()
            p[here, label % V] -= 1.0
            p[~known] = 0.0
            grads.append(torch.einsum("tv,vd->td", p, w) * s["d_loss"][a:a + rows, None].double())
        del lp
    return (torch.cat(losses), torch.cat(grads)) if case["gradient"] else (torch.cat(losses),)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "head_loss":
        return _exact_head(case, s)
    M, K, N, r, L = (case[k] for k in ("M", "K", "N", "r", "L"))
    blank = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    if case["kind"] == "adapters_grad":
        dA, dB = blank(L, r, K), blank(L, N, r)
    else:
        low, out = blank(M, r), s["base"].double()
    for a in range(L):
        mine = torch.nonzero(s["adapter_of"] == a).flatten()
        c, A, B = s["scales"][a].double(), s["A"][a].double(), s["B"][a].double()
        if case["kind"] == "adapters_grad":
            dA[a] = c * torch.einsum("tj,tk->jk", s["G"][mine].double(), s["X"][mine].double())
            dB[a] = c * torch.einsum("tn,tj->nj", s["dY"][mine].double(), s["H"][mine].double())
        elif case["kind"] == "adapters":
            low[mine] = torch.einsum("tk,jk->tj", s["X"][mine].double(), A)
            out[mine] += c * torch.einsum("tj,nj->tn", low[mine], B)
        else:
            low[mine] = torch.einsum("tn,nj->tj", s["dY"][mine].double(), B)
            out[mine] += c * torch.einsum("tj,jk->tk", low[mine], A)
    if case["kind"] == "adapters_grad":
        return dA, dB
    return (out,) if s["low"] is None else (out, low)
