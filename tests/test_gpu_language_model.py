"""The operators of a language model together: through autograd in float32
against 64 bits, and examples/peri_lm.py, its gradients against torch's and its running."""

import importlib.util
import os

import pytest
import torch

import lm_oracle as oracle
import ops_oracle
from paper_2510_05361_amd import ops

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "peri_lm.py")


def example():
    spec = importlib.util.spec_from_file_location("peri_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_step_through_autograd():
    """embedding, a block of norms and two matrices, the tied table as output, cross entropy; then Muon and
    AdamW.  Every operator is within some U of its result; products of 48 terms are off by about 7 U of
    theirs (each way, two in a row, and through four norms), so gradients by less than 200 U of their norm, and 16 times
    that is let pass.  Steps are checked from the gradients that there are, as in the operators' own tests."""
    v, d, rows = 97, 48, 130
    gen = torch.Generator().manual_seed(0)
    start = {"table": torch.randn((v, d), generator=gen), "up": torch.randn((80, d), generator=gen) * d ** -0.5,
             "down": torch.randn((d, 80), generator=gen) * 80 ** -0.5, "post": torch.rand(d, generator=gen) + 0.5,
             "pre0": torch.rand(d, generator=gen) + 0.5, "pre1": torch.rand(d, generator=gen) + 0.5}
    tokens = torch.randint(-1, v, (rows,), generator=gen)
    targets = torch.randint(-1, v, (rows,), generator=gen)

    p = {k: t.cuda().requires_grad_() for k, t in start.items()}
    x = ops.embedding(tokens.cuda(), p["table"], scale=0.7)
    _, n = ops.peri_norm(x, None, None, p["pre0"])
    f = torch.tanh(n @ p["up"].t()) @ p["down"].t()
    x, n = ops.peri_norm(x, f, p["post"], p["pre1"], scale=0.5)
    loss = ops.cross_entropy(n @ p["table"].t(), targets.cuda(), z_loss=1e-3)
    loss.backward()

    q = {k: t.double().requires_grad_() for k, t in start.items()}
    y = oracle.embedding(tokens, q["table"], 0.7)
    f = torch.tanh(ops_oracle.norm(y, q["pre0"], 1e-5, False) @ q["up"].t()) @ q["down"].t()
    _, n = ops_oracle.peri_norm(y, f, q["post"], q["pre1"], None, 1, 0.5, 1e-5, False)
    logits = n @ q["table"].t()
    lse = logits.logsumexp(1)
    each = lse - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0] + 1e-3 * lse.square()
    want = each[targets >= 0].mean()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 100 * oracle.U * float(want.detach())
    for k in start:
        off = (p[k].grad.double().cpu() - q[k].grad).norm()
        assert float(off) < 3200 * oracle.U * float(q[k].grad.norm()), k

    before = {k: t.detach().cpu().double() for k, t in p.items()}
    g = {k: t.grad for k, t in p.items()}
    muon = ops.Muon([p["up"], p["down"]], [g["up"], g["down"]], weight_decay=0.1)
    adamw = ops.AdamW([p[k] for k in ("table", "post", "pre0", "pre1")], [g[k] for k in ("table", "post", "pre0", "pre1")])
    muon.step(0.02)
    adamw.step(1e-3)
    for k in ("up", "down"):
        r, c = before[k].shape
        made, _ = oracle.muon(before[k], g[k].double().cpu(), 0.0, 0.02, 0.95, True, 0.1, max(1.0, r / c) ** 0.5, 5, 1e-7)
        assert float((p[k].detach().double().cpu() - made).norm()) < 8 * oracle.U * float(made.norm()), k
    for k in ("table", "post", "pre0", "pre1"):
        made, _, _ = ops_oracle.adamw(before[k], g[k].double().cpu(), 0.0, 0.0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0)
        assert float((p[k].detach().double().cpu() - made).norm()) < 8 * oracle.U * float(made.norm()), k


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_of_the_example(kind):
    """8-bit products as in test_gpu_example.py, 4 % each; a block's matrices now have three more of them behind
    them, sqrt(13) 4 % = 15 % of a gradient's norm, a cosine of 0.99; 0.92, some two and a half times as much, is let pass."""
    e = example()
    net = e.PeriLM(300, 128, 192, 2, kind)
    p = net.parameters(torch.device("cuda"), 3)
    g = {k: torch.empty_like(v) for k, v in p.items()}
    tokens, targets = e.Text(300, 7, 90, torch.device("cuda"), 4).batch()
    tokens[0, 5:9] = -1
    loss = float(net.loss_and_gradients(p, g, tokens, targets))

    q = {k: v.detach().cpu().requires_grad_() for k, v in p.items()}
    x = oracle.embedding(tokens.cpu(), q["table"], 128 ** 0.5)
    for i in range(2):
        f = torch.relu(ops_oracle.norm(x, q[f"pre{i}"], 1e-5, kind == "layer") @ q[f"up{i}"].t()) @ q[f"down{i}"].t()
        x = x + net.scale * ops_oracle.norm(f, q[f"post{i}"], 1e-5, kind == "layer")
    logits = ops_oracle.norm(x, q["pre2"], 1e-5, kind == "layer") @ q["table"].t()
    lse, y = logits.logsumexp(-1), targets.cpu()
    each = lse - logits.gather(-1, y.clamp(min=0)[..., None])[..., 0] + 1e-4 * lse.square()
    want = each[y >= 0].mean()
    want.backward()
    assert abs(loss - float(want.detach())) < 0.02 * float(want.detach())
    for k in p:
        a, b = g[k].cpu().flatten().double(), q[k].grad.flatten().double()
        assert float(a @ b / (a.norm() * b.norm())) > 0.92, k


def test_the_example_runs():
    losses = example().train(steps=12, say=lambda _: None)
    assert len(losses) == 12 and all(x == x for x in losses)
