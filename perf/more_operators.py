"""The two ends of a language model and the optimizer of its matrices, as timed cases.

    op   "orth"        o = the matrix x with its singular values moved to about 1, by five Newton-Schulz products
         "muon"        one step of the matrices of a GPT with such updates: momentum, orthogonalisation, weight decay
         "embed_fwd"   rows of a table by token, times a scale
         "embed_bwd"   the table's gradient: the rows of each token summed, into a new one or onto one that is there
         "loss"        every token's cross entropy
         "loss_step"   the mean cross entropy and the gradient of the logits

Newton-Schulz, for x [r, c] with r <= c (else its transpose):  X = x / (||x|| + eps), then five times
    A = X X^T,  X = a X + (b A + c A^2) X,   a, b, c = 3.4445, -4.7750, 2.0315.
A token or target below zero stands for none: a row of zeros, no loss, no gradient.
"""

import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_NS, _STEPS, _NS_EPS = (3.4445, -4.7750, 2.0315), 5, 1e-7
_LR, _MOMENTUM, _DECAY = 0.02, 0.95, 0.1
_ALIGN = 64                             # elements between the starts of tensors in one allocation
_LARGEST = {"orth": 6.0e12, "muon": 8.8e12, "embed": 4.8e8, "loss": 3.3e9}  # flops, flops, bytes, bytes: the largest listed case, or less


def listed():
    return [
        # one odd little matrix: the latency of a call
        dict(name="orth_100x37", op="orth", batch=1, r=100, c=37, t="f32"),
        # the up projections of the 16.8M transformer, tall, in one call
        dict(name="orth_4x2048x512_bf16", op="orth", batch=4, r=2048, c=512, t="bf16"),
        # a step of all its matrices
        dict(name="muon_16m", op="muon", d=512, blocks=4, tail="", p="f32", g="f32", nesterov=True),
        # eight blocks of the 1.31B GPT, bf16 gradients
        dict(name="muon_403m", op="muon", d=2048, blocks=8, tail="", p="f32", g="bf16", nesterov=True),
        # decoded tokens of eight requests
        dict(name="embed_fwd_8_tokens", op="embed_fwd", t=8, v=50304, d=2048, w="bf16", y="bf16", none=0.0),
        # eight sequences of 2048 tokens
        dict(name="embed_fwd_16k_tokens", op="embed_fwd", t=16384, v=50304, d=2048, w="bf16", y="bf16", none=0.0),
        # their backward pass, into a fresh gradient of the table
        dict(name="embed_bwd_16k_tokens", op="embed_bwd", t=16384, v=50304, d=2048, y="bf16", none=0.0, onto=False),
        # a padded batch of a small model with a tied table, whose gradient holds the output projection's already
        dict(name="embed_bwd_1999_tied", op="embed_bwd", t=1999, v=50304, d=768, y="bf16", none=0.1, onto=True),
        # the score of a short text
        dict(name="loss_64_tokens", op="loss", t=64, v=8192, x="f32", none=0.0, masked=0),
        # evaluation of two sequences, the last token without a target
        dict(name="loss_4096_tokens", op="loss", t=4096, v=50304, x="bf16", none=0.01, masked=0),
        # an odd vocabulary in fp32 with masked columns, a padded batch
        dict(name="loss_step_2047_f32", op="loss_step", t=2047, v=32003, x="f32", none=0.1, masked=5),
        # a training step of eight sequences
        dict(name="loss_step_16k_tokens", op="loss_step", t=16384, v=50304, x="bf16", none=0.0, masked=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """lo..hi over their logarithm; half of them multiples of 64, half any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


def draw(rng):
    op = rng.choice(("orth", "muon", "embed_fwd", "embed_bwd", "loss", "loss_step"))
    while True:
        if op == "orth":
            c = dict(op=op, batch=_log_int(rng, 1, 32), r=_size(rng, 1, 8192), c=_size(rng, 1, 8192), t=rng.choice(("f32", "bf16")))
        elif op == "muon":
            c = dict(op=op, d=_size(rng, 32, 2048), blocks=_log_int(rng, 1, 8),
                     tail=" ".join(f"{rng.randrange(1, 600)}x{rng.randrange(1, 600)}" for _ in range(rng.randrange(0, 4))),
                     p=rng.choice(("f32", "f32", "bf16")), g=rng.choice(("f32", "bf16")), nesterov=rng.random() < 0.7)
        elif op.startswith("embed"):
            c = dict(op=op, t=_log_int(rng, 1, 32768), v=_log_int(rng, 64, 131072), d=_size(rng, 32, 8192),
                     y=rng.choice(("f32", "bf16")), none=rng.choice((0.0, 0.1)))
            if op == "embed_fwd":
                c["w"] = rng.choice(("f32", "bf16"))
            else:
                c["onto"] = rng.random() < 0.5
        else:
            c = dict(op=op, t=_log_int(rng, 1, 32768), v=_log_int(rng, 64, 131072), x=rng.choice(("f32", "bf16")),
                     none=rng.choice((0.0, 0.1)), masked=rng.choice((0, rng.randrange(1, 50))))
        w = work(c)
        if (w["flops"] if op in ("orth", "muon") else w["bytes"]) <= _LARGEST[op.split("_")[0]]:
            return c


def _matrices(c):
    """The shapes of a GPT's matrices and what follows them."""
    d = c["d"]
    return [s for _ in range(c["blocks"]) for s in ((3 * d, d), (d, d), (4 * d, d), (d, 4 * d))] + [tuple(map(int, s.split("x"))) for s in c["tail"].split()]


def _ns_flops(r, c):
    """Five products with A, b A + c A^2 and X, of symmetric results one half; or, where X is wide, three of them and then two
    on A alone, with two products with X."""
    m, n = min(r, c), max(r, c)
    return min(_STEPS * (3 * m * m * n + m ** 3), 6 * m * m * n + 14 * m ** 3)


def work(case):
    c = case
    if c["op"] == "orth":
        return {"bytes": 2 * c["batch"] * c["r"] * c["c"] * _BYTES[c["t"]], "flops": c["batch"] * _ns_flops(c["r"], c["c"])}
    if c["op"] == "muon":
        shapes = _matrices(c)
        n = sum(a * b for a, b in shapes)
        return {"bytes": n * (2 * _BYTES[c["p"]] + _BYTES[c["g"]] + 8), "flops": sum(_ns_flops(a, b) for a, b in shapes)}
    live = c["t"] - int(c["t"] * c["none"])  # rows with a token
    if c["op"] == "embed_fwd":
        return {"bytes": 4 * c["t"] + c["d"] * (live * _BYTES[c["w"]] + c["t"] * _BYTES[c["y"]]), "flops": live * c["d"]}
    if c["op"] == "embed_bwd":
        # a token comes live * P(token) times on average; onto what is there, only the rows of tokens that come are touched
        some = sum(1 - (1 - math.log1p(1 / i) / math.log(c["v"] + 1)) ** live for i in range(1, c["v"] + 1))
        touched = 2 * some if c["onto"] else c["v"]
        return {"bytes": int(4 * c["t"] + c["d"] * (live * _BYTES[c["y"]] + touched * 4)), "flops": live * c["d"]}
    if c["op"] == "loss":
        return {"bytes": live * c["v"] * _BYTES[c["x"]] + 8 * c["t"], "flops": 4 * live * c["v"]}
    return {"bytes": (live + c["t"]) * c["v"] * _BYTES[c["x"]] + 4 * c["t"], "flops": 7 * live * c["v"]}


# --------------------------------------------------------------- the state


def _embed_scale(c):
    return math.sqrt(c["d"])


def _tokens(c, gen):
    """Frequencies fall with the token's number, as words' do; some places hold no token."""
    u = torch.rand(c["t"], device="cuda", generator=gen, dtype=torch.float64)
    ids = (math.log(c["v"] + 1) * u).exp().sub(1).long().clamp(0, c["v"] - 1)
    none = torch.rand(c["t"], device="cuda", generator=gen) < c["none"]
    return torch.where(none, -1, ids).to(torch.int32)


def _updates(gen, r, c, std):
    """A few strong directions in noise, as gradients of trained models have."""
    k = min(16, r, c)
    strong = torch.randn((r, k), device="cuda", generator=gen) * torch.logspace(0, -1.5, k, device="cuda")
    return std * (torch.randn((r, c), device="cuda", generator=gen) + 2 * (strong @ torch.randn((k, c), device="cuda", generator=gen)))


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "orth":
        s["x"] = torch.stack([_updates(gen, c["r"], c["c"], 1e-3) for _ in range(c["batch"])]).to(_DTYPE[c["t"]])
    elif c["op"] == "muon":
        shapes = _matrices(c)
        at = [0]
        for a, b in shapes:
            at.append(at[-1] + -(-a * b // _ALIGN) * _ALIGN)
        s.update(shapes=shapes, at=at)
        s["p"] = torch.empty(at[-1], device="cuda").normal_(0, 0.02, generator=gen).to(_DTYPE[c["p"]])
        s["g"], s["m"] = torch.zeros(at[-1], device="cuda", dtype=_DTYPE[c["g"]]), torch.zeros(at[-1], device="cuda")
        for (a, b), first in zip(shapes, at):
            s["g"][first:first + a * b] = _updates(gen, a, b, 1e-3).view(-1)
            s["m"][first:first + a * b] = _updates(gen, a, b, 5e-3).view(-1)
    elif c["op"] == "embed_fwd":
        s["tokens"] = _tokens(c, gen)
        s["table"] = torch.empty((c["v"], c["d"]), device="cuda").normal_(0, 0.02, generator=gen).to(_DTYPE[c["w"]])
    elif c["op"] == "embed_bwd":
        s["tokens"] = _tokens(c, gen)
        s["dy"] = torch.empty((c["t"], c["d"]), device="cuda").normal_(0, 1e-3, generator=gen).to(_DTYPE[c["y"]])
        if c["onto"]:
            s["dw"] = torch.empty((c["v"], c["d"]), device="cuda").normal_(0, 1e-2, generator=gen)
    else:
        s["targets"] = _tokens(c, gen)
        x = torch.empty((c["t"], c["v"]), device="cuda").normal_(0, 2, generator=gen)
        # a trained model often has its target high
        x.scatter_add_(1, s["targets"].long().clamp(min=0)[:, None], torch.full((c["t"], 1), 6.0, device="cuda"))
        if c["masked"]:
            x[:, c["v"] - c["masked"]:] = -math.inf
            s["targets"].clamp_(max=c["v"] - c["masked"] - 1)
        s["x"] = x.to(_DTYPE[c["x"]])
    return s


def _parts(s, key):
    """Each matrix of one allocation."""
    return [s[key][first:first + a * b].view(a, b) for (a, b), first in zip(s["shapes"], s["at"])]


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "muon":
        s["parts"] = {key: _parts(s, key) for key in ("p", "g", "m")}
        if own:
            from paper_2510_05361_amd import ops
            s["opt"] = ops.Muon(s["parts"]["p"], s["parts"]["g"], momentum=_MOMENTUM, nesterov=case["nesterov"], weight_decay=_DECAY,
                                steps=_STEPS, eps=_NS_EPS, states={"m": s["parts"]["m"]})
    return s


# ------------------------------------------------------------- in 32 bits


def _newton_schulz(x):
    """x [..., r, c] in fp32."""
    a, b, c = _NS
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2).contiguous()
    x = x / (x.square().sum((-1, -2), keepdim=True).sqrt() + _NS_EPS)
    for _ in range(_STEPS):
        gram = x @ x.transpose(-1, -2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(-1, -2) if tall else x


def _muon(s):
    for p, g, m in zip(*(s["parts"][k] for k in ("p", "g", "m"))):
        m.mul_(_MOMENTUM).add_(g.float())
        u = g.float() + _MOMENTUM * m if s["case"]["nesterov"] else m
        lr = _LR * math.sqrt(max(1.0, p.shape[0] / p.shape[1]))
        p.copy_(p.float() * (1 - _LR * _DECAY) - lr * _newton_schulz(u))


def _embed_fwd(s):
    ids = s["tokens"].long()
    rows = s["table"][ids.clamp(min=0)].float() * _embed_scale(s["case"])
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(_DTYPE[s["case"]["y"]])


def _embed_bwd(s):
    c = s["case"]
    ids = s["tokens"].long()
    dw = s["dw"] if c["onto"] else torch.zeros((c["v"], c["d"]), device="cuda")
    rows = s["dy"].float() * _embed_scale(c)
    dw.index_add_(0, ids.clamp(min=0), torch.where(ids[:, None] >= 0, rows, 0.0))
    return dw


def _loss(s):
    c = s["case"]
    x, ids = s["x"].float(), s["targets"].long()
    e = x - x.amax(1, keepdim=True)
    at = e.gather(1, ids.clamp(min=0)[:, None])
    e = e.exp_()
    total = e.sum(1, keepdim=True)
    losses = torch.where(ids >= 0, (total.log() - at)[:, 0], 0.0)
    if c["op"] == "loss":
        return losses
    counted = (ids >= 0).sum().clamp(min=1)
    weight = torch.where(ids >= 0, 1.0 / counted, 0.0)[:, None]
    e.mul_(weight / total).scatter_add_(1, ids.clamp(min=0)[:, None], -weight)
    return {"loss": losses.sum() / counted, "d": e.to(s["x"].dtype)}


def run(state):
    s = state
    c = s["case"]
    if not own:
        if c["op"] == "orth":
            return _newton_schulz(s["x"].float()).to(s["x"].dtype).contiguous()
        if c["op"] == "muon":
            _muon(s)
            return {"p": s["p"], "m": s["m"]}
        return {"embed_fwd": _embed_fwd, "embed_bwd": _embed_bwd, "loss": _loss, "loss_step": _loss}[c["op"]](s)
    from paper_2510_05361_amd import ops

    if c["op"] == "orth":
        return ops.orthogonalize(s["x"], steps=_STEPS, eps=_NS_EPS)
    if c["op"] == "muon":
        s["opt"].step(_LR)
        return {"p": s["p"], "m": s["m"]}
    if c["op"] == "embed_fwd":
        return ops.embedding(s["tokens"], s["table"], scale=_embed_scale(c), dtype=_DTYPE[c["y"]])
    if c["op"] == "embed_bwd":
        return ops.embedding_backward(s["dy"], s["tokens"], c["v"], scale=_embed_scale(c), dw=s.get("dw"), accumulate=c["onto"])
    if c["op"] == "loss":
        return ops.cross_entropy(s["x"], s["targets"], reduction="none")
    loss, d = ops.cross_entropy_step(s["x"], s["targets"])
    return {"loss": loss, "d": d}


# ------------------------------------------------------------- in 64 bits


def _exact_orth(x):
    """Newton-Schulz of one fp64 matrix."""
    flip = x.shape[0] > x.shape[1]
    y = x.t().contiguous() if flip else x.clone()
    y /= math.sqrt(float((y * y).sum())) + _NS_EPS
    k1, k3, k5 = _NS
    for _ in range(_STEPS):
        g = torch.mm(y, y.t())
        poly = torch.mm(g, g).mul_(k5).add_(g, alpha=k3)
        poly.diagonal().add_(k1)
        y = torch.mm(poly, y)
    return y.t() if flip else y


def _exact_embed_bwd(c, s):
    dw = s["dw"].double() if c["onto"] else torch.zeros((c["v"], c["d"]), dtype=torch.float64, device="cuda")
    use = s["tokens"] >= 0
    order = torch.argsort(s["tokens"][use], stable=True)
    ids, counts = torch.unique_consecutive(s["tokens"][use][order], return_counts=True)
    ends = counts.cumsum(0)
    rows = s["dy"][use][order].double() * _embed_scale(c)
    # sums of each token's rows, one row of every token at a time while many have one, then the rest at once
    for i in range(16):
        has = counts > i
        dw[ids[has].long()] += rows[(ends - counts)[has] + i]
    for j in torch.nonzero(counts > 16).view(-1).tolist():
        dw[int(ids[j])] += rows[int(ends[j] - counts[j]) + 16:int(ends[j])].sum(0)
    return dw


def _exact_loss(c, s):
    t, v = s["x"].shape
    ids, use = s["targets"].long(), s["targets"] >= 0
    losses = torch.zeros(t, dtype=torch.float64, device="cuda")
    d = torch.empty((t, v), dtype=torch.float64, device="cuda") if c["op"] == "loss_step" else None
    n = max(1, int(use.sum()))
    for a in range(0, t, 1024):
        x = s["x"][a:a + 1024].double()
        logs = torch.logsumexp(x, 1)
        rows = torch.arange(x.shape[0], device="cuda")
        at = ids[a:a + 1024].clamp(min=0)
        losses[a:a + 1024] = (logs - x[rows, at]) * use[a:a + 1024]
        if d is not None:
            g = torch.exp(x - logs[:, None])
            g[rows, at] -= 1.0
            d[a:a + 1024] = g * (use[a:a + 1024, None] / n)
    return losses if d is None else {"loss": losses.sum() / n, "d": d}


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "orth":
        return torch.stack([_exact_orth(x.double()) for x in s["x"]])
    if c["op"] == "muon":
        out = {k: s[k].double() for k in ("p", "m")}
        for (a, b), first in zip(s["shapes"], s["at"]):
            cut = slice(first, first + a * b)
            g = s["g"][cut].double().view(a, b)
            m = _MOMENTUM * out["m"][cut].view(a, b) + g
            o = _exact_orth(g + _MOMENTUM * m if c["nesterov"] else m)
            out["m"][cut] = m.reshape(-1)
            out["p"][cut] -= (_LR * _DECAY * out["p"][cut].view(a, b) + _LR * max(1.0, a / b) ** 0.5 * o).reshape(-1)
        return out
    if c["op"] == "embed_fwd":
        rows = s["table"][s["tokens"].long().clamp(min=0)].double() * _embed_scale(c)
        rows[s["tokens"] < 0] = 0
        return rows
    return _exact_embed_bwd(c, s) if c["op"] == "embed_bwd" else _exact_loss(c, s)
