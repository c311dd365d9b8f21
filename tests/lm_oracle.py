"""Embedding, cross entropy and orthogonalised updates in 64 bits, from their
definitions (torch on the CPU; nothing of the library), with bounds of what
fp32 arithmetic may be off by."""

from __future__ import annotations

import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative
NS = (3.4445, -4.7750, 2.0315)


def half_step(dtype) -> float:
    """How far a rounding to dtype moves a value, relative to it."""
    return torch.finfo(dtype).eps / 2


def newton_schulz(x, steps, eps):
    """One matrix, in the type of x."""
    a, b, c = NS
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = x / (x.square().sum().sqrt() + eps)
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if tall else x


def muon(p, g, m, lr, momentum, nesterov, decay, factor, steps, eps):
    """(p, m) after a step, in the type of the arguments."""
    m = momentum * m + g
    u = g + momentum * m if nesterov else m
    return p * (1 - lr * decay) - lr * factor * newton_schulz(u, steps, eps), m


def embedding(tokens, table, scale):
    rows = table.shape[0]
    out = table[tokens.clamp(0, max(rows - 1, 0))] * scale if rows else torch.zeros((*tokens.shape, table.shape[1]), dtype=table.dtype)
    out = torch.where((tokens >= rows)[..., None], torch.full_like(out, math.nan), out)
    return torch.where((tokens < 0)[..., None], torch.zeros_like(out), out)


def embedding_backward(dy, tokens, rows, scale):
    """(dw, bound): fp32 sums of pieces of 32 rows, and of the pieces."""
    dw, mag = torch.zeros((rows, dy.shape[-1]), dtype=torch.float64), torch.zeros((rows, dy.shape[-1]), dtype=torch.float64)
    ids, dy = tokens.reshape(-1), dy.reshape(-1, dy.shape[-1])
    use = (ids >= 0) & (ids < rows)
    dw.index_add_(0, ids[use], dy[use])
    mag.index_add_(0, ids[use], dy[use].abs())
    count = torch.bincount(ids[use], minlength=rows).double()
    adds = count.clamp(max=32) + (count / 32).ceil() + 3
    return dw * scale, adds[:, None] * U * mag * abs(scale)


def cross_entropy(x, targets, z):
    """(losses, bound of their error, gradient of each loss, bound): rows of fp64 logits.
    exp(x - m): the difference is off by U |x - m|, its product with log2 e by 2 U of it, the
    hardware's exponential by 2 U: (3 |x - m| + 2) U.  Sums: 1 U for each addition, at most one
    for each eight of a row's elements in turn by 64 lanes, and twenty across lanes."""
    rows, cols = x.shape
    m = x.amax(1, keepdim=True)
    d = x - m
    e = d.exp()
    s = e.sum(1, keepdim=True)
    p = e / s
    lse = m + s.log()
    at = d.gather(1, targets.clamp(0, cols - 1)[:, None])
    finite = torch.where(d.isfinite(), d.abs(), torch.zeros_like(d))
    rel_s = U * ((p * (3 * finite + 2)).sum(1, keepdim=True) + cols / 64 + 28)
    losses = s.log() - at + z * lse.square()
    err = rel_s + 4 * U * s.log().abs() + 2 * U * at.abs() + z * (4 * U * lse.square() + 2 * lse.abs() * (rel_s + 4 * U * lse.abs())) + 2 * U * losses.abs()
    onehot = torch.zeros_like(x).scatter_(1, targets.clamp(0, cols - 1)[:, None], 1.0)
    grad = p * (1 + 2 * z * lse) - onehot
    gerr = p * (1 + 2 * z * lse.abs()) * ((3 * finite + 12) * U + rel_s + 2 * z * (rel_s + 4 * U * lse.abs())) + 4 * U * onehot + 2.0 ** -120
    live, known = (targets >= 0)[:, None], (targets < cols)[:, None]
    nan, zero = torch.full_like(losses, math.nan), torch.zeros_like(losses)
    losses = torch.where(live, torch.where(known, losses, nan), zero)[:, 0]
    grad = torch.where(live, torch.where(known, grad, nan), zero)
    return losses, torch.where(live, err, zero)[:, 0], grad, torch.where(live, gerr, zero)


def close(got, want, err):
    """Equal where want is not finite, else within err."""
    got = got.double().cpu()
    fine = want.isfinite()
    same = torch.where(fine, (got - want).abs() <= err, (got == want) | (got.isnan() & want.isnan()))
    if not bool(same.all()):
        off = torch.where(fine, (got - want).abs() / (err + 1e-300), torch.zeros_like(want))
        raise AssertionError(f"{int((~same).sum())} of {same.numel()} off, worst {float(off.max()):.3g} times the bound")
