"""Trains a stack of Peri-LN blocks with the operators of
``paper_2510_05361_amd.ops``, first by AdamW, then by MT-DAO.

A block is x' = x + s norm(down(relu(up(norm(x))))): the norms, the residual
scale s and the sum in one pass (``peri_norm``), the linear layers in 8-bit
blocks (``linear8``), the gradients written out by hand with the operators'
backward passes.  The warm-up runs AdamW with 8-bit states over the list of
parameters; its parameters are then the start of K workers, whose local steps
and averaging ``MtdaoOptimizer`` takes, each worker with batches of its own.
The task is synthetic: the outputs of a fixed random two-layer network.

    python examples/peri_blocks.py --warmup 60 --steps 60
"""

from __future__ import annotations

import argparse
import os
import sys
from typing import Dict, List, Tuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_05361_amd import mtdao, ops  # noqa: E402
from paper_2510_05361_amd.optimizer import MtdaoOptimizer  # noqa: E402


class PeriBlocks:
    """The shapes of the parameters, and loss and gradients at given ones."""

    def __init__(self, d: int, hidden: int, blocks: int, kind: str = "rms"):
        self.d, self.blocks, self.kind = d, blocks, kind
        self.scale = blocks ** -0.5
        self.shapes: Dict[str, Tuple[int, ...]] = {"pre0": (d,)}
        for i in range(blocks):
            self.shapes.update({f"up{i}": (hidden, d), f"down{i}": (d, hidden), f"post{i}": (d,), f"pre{i + 1}": (d,)})
        self.numel = sum(torch.Size(s).numel() for s in self.shapes.values())
        self.weights: Dict[str, ops.Weight8] = {}

    def views(self, flat: torch.Tensor) -> Dict[str, torch.Tensor]:
        sizes = [torch.Size(s).numel() for s in self.shapes.values()]
        return {k: v.view(s) for (k, s), v in zip(self.shapes.items(), flat[:self.numel].split(sizes))}

    def start(self, device: torch.device, seed: int) -> torch.Tensor:
        gen = torch.Generator(device=device).manual_seed(seed)
        flat = torch.ones(self.numel, device=device)
        for v in self.views(flat).values():
            if v.dim() == 2:
                v.normal_(0, v.shape[1] ** -0.5, generator=gen)
        return flat

    def _weight(self, name: str, w: torch.Tensor) -> ops.Weight8:
        held = self.weights.get(name)
        if held is None:
            held = self.weights[name] = ops.Weight8(w)
        else:
            held.update(w)
        return held

    def forward(self, p: Dict[str, torch.Tensor], x: torch.Tensor) -> Tuple[torch.Tensor, List[Tuple[torch.Tensor, ...]]]:
        """norm(x of the last block) in bfloat16, and what the backward pass needs."""
        w = {k: self._weight(k, p[k]) for k in self.shapes if len(self.shapes[k]) == 2}
        x, n = ops.peri_norm(x, None, None, p["pre0"], kind=self.kind, branch_dtype=torch.bfloat16)
        kept: List[Tuple[torch.Tensor, ...]] = [(x,)]
        for i in range(self.blocks):
            a = torch.relu(ops.linear8(n, w[f"up{i}"]))
            f = ops.linear8(a, w[f"down{i}"])
            x, after = ops.peri_norm(x, f, p[f"post{i}"], p[f"pre{i + 1}"], kind=self.kind, scale=self.scale)
            kept.append((n, a, f, x))
            n = after
        return n, kept

    def backward(self, p: Dict[str, torch.Tensor], g: Dict[str, torch.Tensor], dn: torch.Tensor, kept: List[Tuple[torch.Tensor, ...]]) -> torch.Tensor:
        """The gradients of the parameters into ``g``; returns that of x."""
        w, dx = self.weights, None
        for i in reversed(range(self.blocks)):
            n, a, f, x = kept.pop()
            dx, df, g[f"post{i}"][:], g[f"pre{i + 1}"][:], _ = ops.peri_norm_backward(dx, dn, x, f, p[f"post{i}"], p[f"pre{i + 1}"], kind=self.kind,
                                                                                     scale=self.scale)
            da, _ = ops.linear8_backward(df, a, w[f"down{i}"], dw=g[f"down{i}"])
            dn, _ = ops.linear8_backward(da * (a > 0), n, w[f"up{i}"], dw=g[f"up{i}"])
        dx, _, _, g["pre0"][:], _ = ops.peri_norm_backward(dx, dn, kept.pop()[0], None, None, p["pre0"], kind=self.kind)
        return dx

    def loss_and_gradients(self, flat: torch.Tensor, grads: torch.Tensor, x: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """Mean square of norm(x of the last block) - target; the gradients of
        ``flat`` go into ``grads`` (both [numel], float32)."""
        p = self.views(flat)
        n, kept = self.forward(p, x)
        off = n.float() - target
        self.backward(p, self.views(grads), (off * (2.0 / off.numel())).bfloat16(), kept)
        return off.square().mean()


class Task:
    """Batches of inputs and what the fixed network makes of them."""

    def __init__(self, d: int, tokens: int, device: torch.device, seed: int):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.tokens, self.d, self.device = tokens, d, device
        teacher = torch.Generator(device=device).manual_seed(7)
        self.a, self.b = (torch.randn((d, d), device=device, generator=teacher) * d ** -0.5 for _ in range(2))

    def batch(self) -> Tuple[torch.Tensor, torch.Tensor]:
        x = torch.randn((self.tokens, self.d), device=self.device, generator=self.gen)
        return x, torch.tanh(x @ self.a) @ self.b


def train(d: int = 256, hidden: int = 512, blocks: int = 2, tokens: int = 1024, workers: int = 2, warmup: int = 60, steps: int = 60,
          lr: float = 3e-3, period: int = 8, say=print) -> List[float]:
    """The losses of the warm-up's steps, then those of MT-DAO's (their mean
    over the workers)."""
    device = torch.device("cuda")
    net = PeriBlocks(d, hidden, blocks)
    flat, grads = net.start(device, 0), torch.empty((workers, net.numel), device=device)
    losses: List[torch.Tensor] = []

    task = Task(d, tokens, device, 1)
    params, of = net.views(flat), net.views(grads[0])
    adamw = ops.AdamW(list(params.values()), list(of.values()), betas=(0.9, 0.95), max_norm=1.0, state_bits=8,
                      weight_decay=[0.01 if v.dim() == 2 else 0.0 for v in params.values()])
    for step in range(warmup):
        losses.append(net.loss_and_gradients(flat, grads[0], *task.batch()))
        adamw.step(lr * min(1.0, (step + 1) / 10))
        if step % 20 == 0:
            say(f"AdamW  step {step:4d}  loss {float(losses[-1]):.4f}")
    adamw.close()

    cfg = mtdao.make_config("adam", replicas=workers, beta1=(0.9, 0.99), omega=(0.5, 0.4), numel=net.numel, beta2=0.95, eps=1e-8,
                            period_x=period, period_u=(2 * period,) * 2, period_v=4 * period)
    opt = MtdaoOptimizer(cfg, device, x0=flat)
    tasks = [Task(d, tokens, device, 2 + k) for k in range(workers)]
    for step in range(steps):
        each = [net.loss_and_gradients(opt.x[k], grads[k], *tasks[k].batch()) for k in range(workers)]
        losses.append(torch.stack(each).mean())
        opt.step_sync(grads, 0.3 * lr)
        if step % 20 == 0:
            say(f"MT-DAO step {step:4d}  loss {float(losses[-1]):.4f}")
    opt.close()
    return torch.stack(losses).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("d", 256), ("hidden", 512), ("blocks", 2), ("tokens", 1024), ("workers", 2), ("warmup", 60), ("steps", 60)):
        ap.add_argument(f"--{name}", type=int, default=value)
    losses = train(**vars(ap.parse_args()))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
