"""The operators of a Peri-LN training step next to the optimizer, as timed cases.

    op   "adamw"        one AdamW step over the tensors of a GPT: states in 32 or 8 bits, weight decay on matrices, optional global-norm clip
         "peri_fwd"     x' = x + scale gate norm(f) w_post;  n = norm(x') w_pre
         "peri_bwd"     the gradients of x, f, w_post, w_pre and gate
         "linear_fwd"   y = x W^T, both in 8-bit floating point with a scale per block of 128
         "linear_bwd"   dx = dy W and dw = dy^T x, likewise
         "linear_step"  both

An 8-bit value is an e4m3 code times its block's power of two 2^e, the smallest with which no finite value of the block exceeds 448.
Blocks are 128 consecutive elements of a tensor (AdamW's states, sqrt(v) in the place of v), 128 elements along the contraction
(activations, gradients) or 128 x 128 (weights).
"""

import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_B = 128                                # elements of a block
_CODE, _SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
_BETA1, _BETA2, _EPS, _LR, _DECAY, _RHO, _START = 0.9, 0.95, 1e-8, 1e-3, 0.1, 1.0, 1000
_NORM_EPS = 1e-5
_SCALE_RES = 0.25                       # residual scale of the block
_LARGEST = {"adamw": 18.6e9, "peri": 4.1e8, "linear": 1.7e12}  # bytes, bytes, flops of the largest listed cases


def listed():
    return [
        # a small model's step: latency of one call over 10 tensors
        dict(name="adamw_32bit_57k", op="adamw", d=64, blocks=1, vocab=128, tail=0, p="f32", g="f32", bits=32, clip=False),
        # a 354M GPT with global-norm clipping, 194 tensors
        dict(name="adamw_32bit_354m_clip", op="adamw", d=1024, blocks=24, vocab=50304, tail=0, p="f32", g="f32", bits=32, clip=True),
        # a 16.8M transformer with a ragged tail tensor, 8-bit states
        dict(name="adamw_8bit_16m_ragged", op="adamw", d=512, blocks=4, vocab=8192, tail=37, p="f32", g="f32", bits=8, clip=True),
        # a 1.31B GPT, bf16 gradients, 8-bit states
        dict(name="adamw_8bit_1311m", op="adamw", d=2048, blocks=24, vocab=50304, tail=0, p="f32", g="bf16", bits=8, clip=False),
        # one token of a served model
        dict(name="peri_fwd_1_token", op="peri_fwd", t=1, d=2048, stream="bf16", branch="bf16", w="bf16", kind="rms", gate="channel", rows=0),
        # eight sequences of 2048 tokens
        dict(name="peri_fwd_16k_tokens", op="peri_fwd", t=16384, d=2048, stream="bf16", branch="bf16", w="bf16", kind="rms", gate="channel",
             rows=0),
        # fp32 residual stream, LayerNorm, a gate for each sequence, the last one cut short
        dict(name="peri_bwd_2047_seq_gate", op="peri_bwd", t=2047, d=768, stream="f32", branch="bf16", w="f32", kind="layer", gate="seq",
             rows=512),
        # the backward pass of eight sequences
        dict(name="peri_bwd_16k_tokens", op="peri_bwd", t=16384, d=2048, stream="bf16", branch="bf16", w="bf16", kind="rms", gate="channel",
             rows=0),
        # eight decoded tokens through an up projection
        dict(name="linear_fwd_8_tokens", op="linear_fwd", m=8, n=8192, k=2048, x="bf16"),
        # a ragged batch through the QKV projection of d = 768
        dict(name="linear_fwd_1999_tokens", op="linear_fwd", m=1999, n=2304, k=768, x="bf16"),
        # the gradients of a narrow layer: few tiles, a long contraction for dw
        dict(name="linear_bwd_d512", op="linear_bwd", m=8191, n=1536, k=512, x="bf16"),
        # forward and backward of the up projection of the 1.31B model over 16k tokens
        dict(name="linear_step_16k_tokens", op="linear_step", m=16384, n=8192, k=2048, x="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """lo..hi over their logarithm; half of them whole blocks, half any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.5 else max(_B, v // _B * _B)


def draw(rng):
    op = rng.choice(("adamw", "adamw", "peri_fwd", "peri_bwd", "linear_fwd", "linear_bwd", "linear_step"))
    while True:
        if op == "adamw":
            c = dict(op=op, d=_log_int(rng, 32, 2048), blocks=_log_int(rng, 1, 24), vocab=_log_int(rng, 64, 50304),
                     tail=rng.choice((0, rng.randrange(1, 1000))), p=rng.choice(("f32", "f32", "bf16")), g=rng.choice(("f32", "bf16")),
                     bits=rng.choice((8, 32)), clip=rng.random() < 0.5)
        elif op.startswith("peri"):
            c = dict(op=op, t=_log_int(rng, 1, 16384), d=_size(rng, 64, 8192), w=rng.choice(("f32", "bf16")),
                     kind=rng.choice(("rms", "rms", "layer")), gate=rng.choice(("none", "channel", "seq")), rows=0)
            c["stream"], c["branch"] = rng.choice((("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")))
            if c["gate"] == "seq":
                c["rows"] = _log_int(rng, 1, c["t"])
        else:
            c = dict(op=op, m=_size(rng, 1, 16384) if rng.random() < 0.8 else rng.randrange(1, 65), n=_size(rng, 64, 8192),
                     k=_size(rng, 64, 8192), x=rng.choice(("bf16", "bf16", "f32")))
        w = work(c)
        if (w["flops"] if op.startswith("linear") else w["bytes"]) <= _LARGEST[op.split("_")[0]]:
            return c


def _tensors(c):
    """Elements of the tensors, those with weight decay (matrices) first, and how many these are."""
    d = c["d"]
    mats = [c["vocab"] * d] + [a * d * d for _ in range(c["blocks"]) for a in (3, 1, 4, 4)]
    return mats + [d] * (4 * c["blocks"] + 1) + ([c["tail"]] if c["tail"] else []), len(mats)


def _gates(c):
    return {"none": 0, "channel": 1}.get(c["gate"], -(-c["t"] // max(1, c["rows"])))


def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(_tensors(c)[0])
        held = 16 if c["bits"] == 32 else 4 + 4 / _B
        return {"bytes": int(n * (2 * _BYTES[c["p"]] + _BYTES[c["g"]] * (2 if c["clip"] else 1) + held)), "flops": 14 * n}
    if c["op"].startswith("peri"):
        td, s, b = c["t"] * c["d"], _BYTES[c["stream"]], _BYTES[c["branch"]]
        rows = (2 + _gates(c)) * c["d"]
        if c["op"] == "peri_fwd":
            return {"bytes": td * 2 * (s + b) + rows * _BYTES[c["w"]], "flops": 12 * td}
        return {"bytes": td * 3 * (s + b) + rows * (_BYTES[c["w"]] + 4), "flops": 32 * td}
    m, n, k, e = c["m"], c["n"], c["k"], _BYTES[c["x"]]
    fwd = {"bytes": e * m * (k + n) + n * k, "flops": 2 * m * n * k}
    bwd = {"bytes": e * m * (2 * k + n) + n * k + 4 * n * k, "flops": 4 * m * n * k}
    if c["op"] == "linear_fwd":
        return fwd
    if c["op"] == "linear_bwd":
        return bwd
    return {"bytes": e * m * (2 * k + 2 * n) + 5 * n * k, "flops": fwd["flops"] + bwd["flops"]}


# ------------------------------------------------------------- in 32 bits


def _blocks(x, dims):
    """e4m3 codes and e8m0 scales of fp32 blocks that span `dims`."""
    a = x.abs()
    bits = torch.where(a.isfinite(), a, 0.0).amax(dims, keepdim=True).view(torch.int32)
    e = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp(1, 254)
    codes = (x * ((254 - e) << 23).view(torch.float32)).to(_CODE)
    return codes, e.to(torch.uint8).view(_SCALE)


def _blocks_root(v):
    """_blocks of sqrt(v); no positive value becomes 0."""
    r = v.sqrt()
    codes, scale = _blocks(r, -1)
    return torch.where((r > 0) & (codes.float() == 0), 2.0 ** -9, codes.float()).to(_CODE), scale


def _along_rows(x):
    """The values that x [r, c] has with blocks of 128 along its rows, zeros up to whole blocks."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % _B))
    codes, scale = _blocks(x.view(x.shape[0], -1, _B), -1)
    return (codes.float() * scale.float()).view(x.shape)


def _weight(w):
    """Codes [n, k] padded to whole blocks and scales [n/128, 1, k/128, 1]."""
    w = torch.nn.functional.pad(w.float(), (0, -w.shape[1] % _B, 0, -w.shape[0] % _B))
    codes, scale = _blocks(w.view(w.shape[0] // _B, _B, -1, _B), (1, 3))
    return codes, scale


def _weight_values(codes, scale, n, k):
    w = codes.float() * scale.float()
    return w.view(w.shape[0] * _B, -1)[:n, :k]


def _adamw(s):
    c = s["case"]
    s["step"] += 1
    g = s["g"].float()
    if c["clip"]:
        g = g * (_RHO / g.square().sum().sqrt()).clamp(max=1.0)
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, _B) * s["m_scale"].float()[:, None]).view(-1)
        v = (s["v"].float().view(-1, _B) * s["v_scale"].float()[:, None]).view(-1).square()
    m.mul_(_BETA1).add_(g, alpha=1 - _BETA1)
    v.mul_(_BETA2).addcmul_(g, g, value=1 - _BETA2)
    update = m / ((v / (1 - _BETA2 ** s["step"])).sqrt() + _EPS)
    p = s["p"].float()
    p[:s["decayed"]].mul_(1 - _LR * _DECAY)
    p.sub_(update, alpha=_LR / (1 - _BETA1 ** s["step"]))
    if p is not s["p"]:
        s["p"].copy_(p)
    if c["bits"] == 8:
        for key, made in (("m", _blocks(m.view(-1, _B), -1)), ("v", _blocks_root(v.view(-1, _B)))):
            s[key].copy_(made[0].view(-1))
            s[key + "_scale"].copy_(made[1].view(-1))


def _unit(c, z):
    """(z - mean) r and r of every row."""
    if c["kind"] == "layer":
        z = z - z.mean(-1, keepdim=True)
    r = (z.square().mean(-1, keepdim=True) + _NORM_EPS).rsqrt()
    return z * r, r


def _through(c, y, zh, r):
    """The gradient of z for the gradient y of its normalized row."""
    t = y - zh * (y * zh).mean(-1, keepdim=True)
    return r * (t - y.mean(-1, keepdim=True) if c["kind"] == "layer" else t)


def _gate_rows(s):
    """The gate of every row times the residual scale."""
    c = s["case"]
    if c["gate"] == "none":
        return _SCALE_RES
    gate = s["gate"].float() * _SCALE_RES
    return gate if c["gate"] == "channel" else gate.repeat_interleave(c["rows"], 0)[:c["t"]]


def _peri_fwd(s):
    c = s["case"]
    x = s["x"].float() + _gate_rows(s) * (_unit(c, s["f"].float())[0] * s["w_post"].float())
    n = _unit(c, x)[0] * s["w_pre"].float()
    return {"x": x.to(s["x"].dtype), "n": n.to(s["f"].dtype)}


def _peri_bwd(s):
    c = s["case"]
    gate, w_post, w_pre = _gate_rows(s), s["w_post"].float(), s["w_pre"].float()
    xh, xr = _unit(c, s["x"].float())
    fh, fr = _unit(c, s["f"].float())
    dn = s["dn"].float()
    dx = s["dx"].float() + _through(c, dn * w_pre, xh, xr)
    dh = dx * gate
    out = {"x": dx.to(s["x"].dtype), "f": _through(c, dh * w_post, fh, fr).to(s["f"].dtype), "w_pre": (dn * xh).sum(0),
           "w_post": (dh * fh).sum(0)}
    if c["gate"] != "none":
        each = dx * (fh * w_post) * _SCALE_RES
        if c["gate"] == "seq":
            each = torch.nn.functional.pad(each, (0, 0, 0, -c["t"] % c["rows"])).view(-1, c["rows"], c["d"]).sum(1)
        else:
            each = each.sum(0, keepdim=True)
        out["gate"] = each
    return out


def _linear(s):
    c, out = s["case"], {}
    w = _weight_values(*s["weight"], c["n"], c["k"])
    x = s["x"]
    if c["op"] != "linear_bwd":
        out["y"] = (_along_rows(x)[:, :c["k"]] @ w.t()).to(x.dtype)
    if c["op"] != "linear_fwd":
        dy = s["dy"]
        out["dx"] = (_along_rows(dy)[:, :c["n"]] @ w).to(x.dtype)
        out["dw"] = _along_rows(dy.t()) @ _along_rows(x.t()).t()
    return out


# --------------------------------------------------------------- the state


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype="f32", mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=gen).to(_DTYPE[dtype])

    s = {"case": c}
    if c["op"] == "adamw":
        # tensors at whole blocks of one allocation each, in the middle of a run
        numels, mats = _tensors(c)
        at = [0]
        for n in numels:
            at.append(at[-1] + -(-n // _B) * _B)
        total = at[-1]
        std = 1e-3 if c["clip"] else 1e-4
        s.update(numels=numels, at=at, decayed=at[mats], step=_START)
        s["p"], s["g"] = normal(total, 0.02, c["p"]), normal(total, std, c["g"])
        m = normal(total, std * math.sqrt((1 - _BETA1) / (1 + _BETA1)))
        v = torch.empty(total, device="cuda").uniform_(0.5, 1.5, generator=gen).mul_(std * std)
        for n, a, b in zip(numels, at, at[1:]):
            if a + n < b:
                for t in (s["p"], s["g"], m, v):
                    t[a + n:b] = 0
        if c["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            for key, (codes, scale) in (("m", _blocks(m.view(-1, _B), -1)), ("v", _blocks_root(v.view(-1, _B)))):
                s[key], s[key + "_scale"] = codes.view(-1), scale.view(-1)
    elif c["op"].startswith("peri"):
        t, d = c["t"], c["d"]
        # a few channels of the stream are much larger than the rest, as in trained models
        s["x"] = (normal((t, d), 1.0) * (1 + 8 * (torch.rand(d, device="cuda", generator=gen) < 0.01))).to(_DTYPE[c["stream"]])
        s["f"] = normal((t, d), 0.3, c["branch"], 0.05)
        s["w_post"], s["w_pre"] = normal(d, 0.1, c["w"], 1.0), normal(d, 0.1, c["w"], 1.0)
        s["gate"] = normal((_gates(c), d), 0.3, c["w"], 0.5) if c["gate"] != "none" else None
        if c["op"] == "peri_bwd":
            s["dx"], s["dn"] = normal((t, d), 1e-3, c["stream"]), normal((t, d), 1e-3, c["branch"])
    else:
        m, n, k = c["m"], c["n"], c["k"]
        s["x"] = (normal((m, k), 1.0) * (1 + 8 * (torch.rand(k, device="cuda", generator=gen) < 0.01))).to(_DTYPE[c["x"]])
        s["w"] = normal((n, k), 0.02, "bf16")
        if c["op"] != "linear_fwd":
            s["dy"] = (normal((m, n), 1e-3) * torch.rand((m, 1), device="cuda", generator=gen)).to(_DTYPE[c["x"]])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adamw" and own:
        from paper_2510_05361_amd import ops

        def parts(t, per=1):
            return [t[a // per:a // per + -(-n // per)] for a, n in zip(s["at"], s["numels"])]

        held = {"m": parts(s["m"]), "v": parts(s["v"])}
        if case["bits"] == 8:
            held.update(m_scale=parts(s["m_scale"], _B), v_scale=parts(s["v_scale"], _B))
        mats = _tensors(case)[1]
        s["opt"] = ops.AdamW(parts(s["p"]), parts(s["g"]), betas=(_BETA1, _BETA2), eps=_EPS,
                             weight_decay=[_DECAY] * mats + [0.0] * (len(s["numels"]) - mats), max_norm=_RHO if case["clip"] else 0.0,
                             state_bits=case["bits"], start_step=_START, states=held)
    elif case["op"].startswith("linear"):
        s["weight"] = _weight(s["w"])
        if own:
            from paper_2510_05361_amd import ops
            s["weight8"] = ops.Weight8(s["w"])
    return s


def run(state):
    s = state
    c = s["case"]
    if c["op"] == "adamw":
        if own:
            s["opt"].step(_LR)
        else:
            _adamw(s)
        return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale") if k in s}
    if not own:
        return _peri_fwd(s) if c["op"] == "peri_fwd" else _peri_bwd(s) if c["op"] == "peri_bwd" else _linear(s)
    from paper_2510_05361_amd import ops

    if c["op"].startswith("peri"):
        how = dict(gate=s["gate"], rows_per_gate=c["rows"], scale=_SCALE_RES, eps=_NORM_EPS, kind=c["kind"])
        if c["op"] == "peri_fwd":
            x, n = ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"], **how)
            return {"x": x, "n": n}
        dx, df, dw_post, dw_pre, dgate = ops.peri_norm_backward(s["dx"], s["dn"], s["x"], s["f"], s["w_post"], s["w_pre"], **how)
        out = {"x": dx, "f": df, "w_pre": dw_pre, "w_post": dw_post}
        if dgate is not None:
            out["gate"] = dgate
        return out
    out = {}
    if c["op"] != "linear_bwd":
        out["y"] = ops.linear8(s["x"], s["weight8"])
    if c["op"] != "linear_fwd":
        out["dx"], out["dw"] = ops.linear8_backward(s["dy"], s["x"], s["weight8"])
    return out


# ------------------------------------------------------------- in 64 bits


def _two_to(e):
    """2^e in fp64 for whole e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _held(x, dims):
    """Codes and scales, as fp64 values, of fp64 blocks that span `dims`."""
    fraction, exponent = torch.frexp(x.abs().amax(dims, keepdim=True))
    e = exponent - 9 + (2 * fraction > 1.75).to(exponent.dtype)
    e = torch.where(fraction == 0, -126, e).clamp(-126, 127)
    y = x * _two_to(-e)
    step = _two_to(torch.frexp(y)[1].sub_(1).clamp_(min=-6).sub_(3))
    return torch.round(y / step) * step, _two_to(e)


def _held_rows(x):
    x = torch.nn.functional.pad(x.double(), (0, -x.shape[1] % _B))
    codes, scale = _held(x.view(x.shape[0], -1, _B), -1)
    return (codes * scale).view(x.shape)


def _exact_adamw(c, s):
    b1, b2, eps, lr, wd, t = _BETA1, _BETA2, _EPS, _LR, _DECAY, _START + 1
    total, cols = s["p"].numel(), 1 << 26
    clip = 1.0
    if c["clip"]:
        clip = min(1.0, _RHO / math.sqrt(sum(float(a.double().square().sum()) for a in s["g"].split(cols))))
    eight = c["bits"] == 8
    keys = ("p", "m", "v", "m_scale", "v_scale") if eight else ("p", "m", "v")
    out = {k: torch.empty(s[k].shape, dtype=torch.float64, device="cuda") for k in keys}
    for at in range(0, total, cols):
        cut, few = slice(at, min(total, at + cols)), slice(at // _B, min(total, at + cols) // _B)
        g, m, v, p = (s[k][cut].double() for k in ("g", "m", "v", "p"))
        g = g * clip
        if eight:
            m = (m.view(-1, _B) * s["m_scale"][few].double()[:, None]).view(-1)
            v = (v.view(-1, _B) * s["v_scale"][few].double()[:, None]).view(-1) ** 2
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        p[:max(0, s["decayed"] - at)] *= 1 - lr * wd
        out["p"][cut] = p - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
        if eight:
            codes, scale = _held(m.view(-1, _B), -1)
            out["m"][cut], out["m_scale"][few] = codes.view(-1), scale.view(-1)
            codes, scale = _held(v.sqrt().view(-1, _B), -1)
            codes = torch.where((codes == 0) & (v.view(-1, _B) > 0), 2.0 ** -9, codes)
            out["v"][cut], out["v_scale"][few] = codes.view(-1), scale.view(-1)
        else:
            out["m"][cut], out["v"][cut] = m, v
    return out


def _exact_norm(c, z, w):
    mean = z.mean(-1, keepdim=True) if c["kind"] == "layer" else 0.0
    return (z - mean) / torch.sqrt(((z - mean) ** 2).mean(-1, keepdim=True) + _NORM_EPS) * w


def _exact_peri(c, s):
    get = {k: (s[k].double() if s[k] is not None else None) for k in ("x", "f", "w_post", "w_pre", "gate")}

    def branch(f, w_post, gate):
        h = _SCALE_RES * _exact_norm(c, f, w_post)
        if gate is None:
            return h
        each = torch.arange(c["t"], device="cuda") // (c["rows"] if c["gate"] == "seq" else c["t"])
        return h * gate[each]

    if c["op"] == "peri_fwd":
        x = get["x"] + branch(get["f"], get["w_post"], get["gate"])
        return {"x": x, "n": _exact_norm(c, x, get["w_pre"])}
    for v in get.values():
        if v is not None:
            v.requires_grad_()
    x, w_pre = torch.autograd.grad((_exact_norm(c, get["x"], get["w_pre"]) * s["dn"].double()).sum(), (get["x"], get["w_pre"]))
    x = x + s["dx"].double()
    into = [k for k in ("f", "w_post", "gate") if get[k] is not None]
    grads = torch.autograd.grad((branch(get["f"], get["w_post"], get["gate"]) * x).sum(), [get[k] for k in into])
    return {"x": x, "w_pre": w_pre, **dict(zip(into, grads))}


def _exact_linear(c, s):
    n, k = c["n"], c["k"]
    w = torch.nn.functional.pad(s["w"].double(), (0, -k % _B, 0, -n % _B))
    codes, scale = _held(w.view(w.shape[0] // _B, _B, -1, _B), (1, 3))
    w = (codes * scale).view(w.shape)[:n, :k]
    out = {}
    if c["op"] != "linear_bwd":
        out["y"] = _held_rows(s["x"])[:, :k] @ w.t()
    if c["op"] != "linear_fwd":
        out["dx"] = _held_rows(s["dy"])[:, :n] @ w
        out["dw"] = _held_rows(s["dy"].t()) @ _held_rows(s["x"].t()).t()
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, s)
    return _exact_peri(case, s) if case["op"].startswith("peri") else _exact_linear(case, s)
