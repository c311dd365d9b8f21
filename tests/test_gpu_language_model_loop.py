"""The loop of examples/peri_lm.py: what a step changes and which way, and that nothing of an earlier
step is taken for the present one's."""

import pytest
import torch

from test_gpu_language_model import example

pytestmark = pytest.mark.gpu


def run(monkeypatch, steps):
    """(losses, parameters at the start, after the steps, gradients of the last) of the example's own loop."""
    e, seen = example(), {}
    made, graded = e.PeriLM.parameters, e.PeriLM.loss_and_gradients

    def parameters(self, *args):
        p = made(self, *args)
        seen.update(p=p, start={k: v.clone() for k, v in p.items()})
        return p

    def loss_and_gradients(self, p, g, *batch):
        loss = graded(self, p, g, *batch)
        seen.update(net=self, batch=batch, g={k: v.clone() for k, v in g.items()})
        return loss

    monkeypatch.setattr(e.PeriLM, "parameters", parameters)
    monkeypatch.setattr(e.PeriLM, "loss_and_gradients", loss_and_gradients)
    losses = e.train(steps=steps, say=lambda _: None)
    return e, losses, seen


def test_the_first_step_goes_against_the_gradient(monkeypatch):
    """An orthogonalised update o of u = 1.95 g has <o, g> > 0: it has g's singular vectors, and each singular value s > 0
    becomes a product of s and factors a + b s^2 + c s^4 >= 0.63.  AdamW's first update is g over its own size."""
    _, losses, seen = run(monkeypatch, 1)
    assert len(losses) == 1 and abs(losses[0]) < float("inf")
    for k, now in seen["p"].items():
        g, start = seen["g"][k].double(), seen["start"][k].double()
        matrix = now.dim() == 2 and k != "table"
        lr, decay = (0.02, 0.01) if matrix else (0.002, 0.0)
        change = now.double() - start * (1 - lr * decay)
        assert bool(now.isfinite().all()) and float(g.norm()) > 0, k
        assert float((change * g).sum()) < 0, k


def test_every_parameter_moves_and_losses_are_finite(monkeypatch):
    _, losses, seen = run(monkeypatch, 6)
    assert len(losses) == 6 and all(abs(x) < float("inf") for x in losses)
    for k, now in seen["p"].items():
        assert bool(now.isfinite().all()) and not torch.equal(now, seen["start"][k]), k


def test_weights_in_8_bits_are_the_present_ones(monkeypatch):
    """After the loop's steps its model and a new one over the same parameters give the same loss and gradients, bit for bit."""
    e, _, seen = run(monkeypatch, 4)
    old, p = seen["net"], seen["p"]
    new = e.PeriLM(old.vocab, old.d, old.shapes["up0"][0], old.blocks, old.kind)
    results = []
    for net in (old, new):
        g = {k: torch.empty_like(v) for k, v in p.items()}
        results.append((float(net.loss_and_gradients(p, g, *seen["batch"])), g))
    assert results[0][0] == results[1][0]
    assert all(torch.equal(results[0][1][k], results[1][1][k]) for k in p)
