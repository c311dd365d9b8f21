"""The operators of include/mtdao_ops.h in 64 bits, from their definitions
(torch on the CPU; nothing of the library)."""

from __future__ import annotations

import math

import torch

BLOCK = 128


def two_to(e):
    """2^e in fp64 for whole e in [-1022, 1023]."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def floor_log2(x):
    """floor(log2 |x|) of finite fp64 x != 0 (0 gives a very small number)."""
    m, e = torch.frexp(x.abs())
    return torch.where(m == 0, torch.full_like(e, -2000), e - 1)


def block_exponent(amax):
    """e of the smallest 2^e with amax / 2^e <= 448, clamped to [-126, 127]."""
    f = floor_log2(amax)
    over = amax > 1.75 * two_to(f.clamp(min=-1000))
    e = f - 8 + over.to(f.dtype)
    return e.clamp(-126, 127)


def to_e4m3(y):
    """fp64 values of magnitude at most 448 rounded to e4m3, ties to even."""
    step = two_to(floor_log2(y).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def blocks(x):
    """(codes, e) of the blocks [..., 128] of fp64 x; non-finite values give NaN codes."""
    fine = torch.where(x.isfinite(), x, torch.zeros((), dtype=x.dtype))
    e = block_exponent(fine.abs().amax(-1, keepdim=True))
    return torch.where(x.isfinite(), to_e4m3(fine * two_to(-e)), math.nan), e


def pad_to(x, *multiples):
    """x zero-padded at the end of its last axes to multiples."""
    pads = []
    for size, m in zip(reversed(x.shape), reversed(multiples)):
        pads += [0, -size % m]
    return torch.nn.functional.pad(x, pads)


def rows8(x):
    """(codes [r, kp], e [r, kb]) of x [r, c] in blocks of 1 x 128."""
    x = pad_to(x.double(), BLOCK)
    codes, e = blocks(x.view(x.shape[0], x.shape[1] // BLOCK, BLOCK))
    return codes.view(x.shape), e[..., 0]


def square8(w):
    """(codes [np, kp], e [nb, kb]) of w [n, k] in blocks of 128 x 128."""
    w = pad_to(w.double(), BLOCK, BLOCK)
    n, k = w.shape
    b = w.view(n // BLOCK, BLOCK, k // BLOCK, BLOCK).permute(0, 2, 1, 3).reshape(n // BLOCK, k // BLOCK, BLOCK * BLOCK)
    codes, e = blocks(b)
    return codes.view(n // BLOCK, k // BLOCK, BLOCK, BLOCK).permute(0, 2, 1, 3).reshape(n, k), e[..., 0]


def values(codes, e, scale_rows=1):
    """codes [r, kp] times their scales."""
    s = two_to(e).repeat_interleave(scale_rows, 0)[:codes.shape[0]]
    return (codes.view(codes.shape[0], -1, BLOCK) * s[:, :, None]).view(codes.shape)


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay, clip):
    """(p, m, v) after step t, all fp64; clip: the factor of the gradients."""
    g = g * clip
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps)
    return p, m, v


def clip_factor(grads, max_norm):
    if max_norm <= 0:
        return 1.0
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return min(1.0, max_norm / norm) if norm > 0 else 1.0


def norm(z, w, eps, layer):
    mean = z.mean(-1, keepdim=True) if layer else 0.0
    return (z - mean) / ((z - mean).square().mean(-1, keepdim=True) + eps).sqrt() * w


def peri_norm(x, f, w_post, w_pre, gate, rows_per_gate, scale, eps, layer):
    """(x', n) of fp64 [T, D] inputs; None where an input is missing."""
    out = x
    if f is not None:
        h = norm(f, w_post, eps, layer)
        if gate is not None:
            h = h * gate[torch.arange(x.shape[0]) // rows_per_gate]
        out = x + scale * h
    return out, norm(out, w_pre, eps, layer) if w_pre is not None else None


def peri_norm_backward(d_out, dn, x_out, f, w_post, w_pre, gate, rows_per_gate, scale, eps, layer):
    """Gradients by differentiating the definition: n as a function of x',
    then x' as a function of f and its weights.  Returns a dict."""
    x_out = x_out.clone().requires_grad_()
    out, d = {}, torch.zeros_like(x_out) if d_out is None else d_out
    if w_pre is not None:
        w_pre = w_pre.clone().requires_grad_()
        n = norm(x_out, w_pre, eps, layer)
        gx, out["w_pre"] = torch.autograd.grad((n * (torch.zeros_like(n) if dn is None else dn)).sum(), (x_out, w_pre))
        d = d + gx
    out["x"] = d.detach()
    if f is not None:
        leaves = {"f": f, "w_post": w_post, **({"gate": gate} if gate is not None else {})}
        leaves = {k: t.clone().requires_grad_() for k, t in leaves.items()}
        made, _ = peri_norm(torch.zeros_like(out["x"]), leaves["f"], leaves["w_post"], None, leaves.get("gate"),
                            rows_per_gate, scale, eps, layer)
        out.update(zip(leaves, torch.autograd.grad((made * out["x"]).sum(), list(leaves.values()))))
    return out
