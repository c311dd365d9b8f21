"""Derivatives in forward mode: the operators do not give them, and say so (CPU: what is
refused is refused before a device is looked at)."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2510_05361_amd import ops

X, W, IDS = torch.randn(4, 128), torch.randn(128), torch.zeros(4, dtype=torch.int64)

CALLS = {
    "peri_norm x": (X, lambda t: ops.peri_norm(t, None, None, W)),
    "peri_norm f": (X, lambda t: ops.peri_norm(X, t, W, W)),
    "peri_norm w_post": (W, lambda t: ops.peri_norm(X, X, t, W)),
    "peri_norm w_pre": (W, lambda t: ops.peri_norm(X, None, None, t)),
    "peri_norm gate": (W, lambda t: ops.peri_norm(X, X, W, W, gate=t[None])),
    "linear8 x": (X, lambda t: ops.linear8(t, ops.Weight8.__new__(ops.Weight8))),
    "Weight8": (X, lambda t: ops.Weight8(t)),
    "Weight8.update": (X, lambda t: ops.Weight8.__new__(ops.Weight8).update(t)),
    "embedding": (X, lambda t: ops.embedding(IDS, t)),
    "cross_entropy": (X, lambda t: ops.cross_entropy(t, IDS)),
    "orthogonalize": (X, lambda t: ops.orthogonalize(t)),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("requires_grad", [False, True])
def test_tangents_are_refused(call, requires_grad):
    x, go = CALLS[call]
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x.clone().requires_grad_(requires_grad), torch.ones_like(x))
        with pytest.raises(ValueError, match="requires a gradient|has a tangent" if call == "orthogonalize" else "has a tangent"):
            go(dual)
        with torch.no_grad(), pytest.raises(ValueError, match="has a tangent"):
            go(dual)


@pytest.mark.parametrize("call", ["embedding", "cross_entropy", "orthogonalize"])
def test_tangents_of_function_transforms_are_refused(call):
    x, go = CALLS[call]
    with pytest.raises(ValueError, match="has a tangent"):
        torch.func.jvp(go, (x,), (torch.ones_like(x),))


@pytest.mark.parametrize("call", ["peri_norm x", "Weight8", "embedding", "cross_entropy", "orthogonalize"])
def test_tensors_without_a_tangent_go_on(call):
    """As far as the look at their device."""
    x, go = CALLS[call]
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for t in (x.clone(), dual.detach()):
            with pytest.raises(ValueError, match="the GPU only"):
                go(t)
