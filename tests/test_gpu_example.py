"""examples/peri_blocks.py: its gradients against torch's in float32, and its
training."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "peri_blocks.py")


def example():
    spec = importlib.util.spec_from_file_location("peri_blocks", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients(kind):
    """Codes of e4m3 are off by 2^-4 / sqrt(3) of a value at most in the mean
    square, 4 % with both factors of a product (the step is a sixteenth to an
    eighth of a value): with two products each way in each of two blocks, and
    a third for a weight, gradients are off by sqrt(10) 4 % = 13 % of their
    norm, a cosine of 0.99; three times as much is let pass, 0.92."""
    e = example()
    net = e.PeriBlocks(192, 320, 2, kind)
    flat = net.start(torch.device("cuda"), 3)
    grads = torch.empty_like(flat)
    x, target = e.Task(192, 700, torch.device("cuda"), 4).batch()
    loss = float(net.loss_and_gradients(flat, grads, x, target))

    p = {k: v.cpu().requires_grad_() for k, v in net.views(flat).items()}

    def norm(z, w):
        if kind == "layer":
            z = z - z.mean(-1, keepdim=True)
        return z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w

    y = x.cpu()
    for i in range(2):
        f = torch.relu(norm(y, p[f"pre{i}"]) @ p[f"up{i}"].t()) @ p[f"down{i}"].t()
        y = y + net.scale * norm(f, p[f"post{i}"])
    want = (norm(y, p["pre2"]) - target.cpu()).square().mean()
    want.backward()
    want = float(want.detach())
    assert abs(loss - want) < 0.02 * want
    for k, g in net.views(grads).items():
        a, b = g.cpu().flatten().double(), p[k].grad.flatten().double()
        assert float(a @ b / (a.norm() * b.norm())) > 0.92, k


def test_training():
    losses = example().train(warmup=60, steps=40, say=lambda _: None)
    assert len(losses) == 100 and all(x == x for x in losses)
    start, warm, end = losses[0], sum(losses[50:60]) / 10, sum(losses[-10:]) / 10
    assert warm < 0.6 * start and end < warm


def test_backward_passes_over_changed_tensors_are_refused():
    """What the operators write in place has changed for autograd too."""
    from paper_2510_05361_amd import ops

    x, w = torch.randn((6, 64), device="cuda"), torch.ones(64, device="cuda", requires_grad=True)
    _, n = ops.peri_norm(x, None, None, w)
    ops.AdamW([w.detach()], [torch.ones_like(w)]).step(1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        n.sum().backward()
    a, b = ops.quantize8(torch.randn((6, 256), device="cuda")), ops.quantize8(torch.randn((64, 256), device="cuda"))
    for change in (lambda t: ops.product8(a, b, out=t),
                   lambda t: ops.linear8_backward(torch.ones((3, 6), device="cuda"), torch.ones((3, 64), device="cuda"),
                                                  ops.Weight8(torch.ones((6, 64), device="cuda")), dw=t)):
        y = torch.ones((6, 64), device="cuda")
        s = (y * w).sum()
        change(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            s.backward()
    with torch.inference_mode():
        x = torch.ones((6, 64), device="cuda")
    ops.product8(a, b, out=x)
    opt = ops.AdamW([x], [torch.ones_like(x)])
    opt.step(1e-3)
    assert opt.step_count == 1
