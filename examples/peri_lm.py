"""Trains a small language model of Peri-LN blocks: ``Muon`` for the blocks'
matrices, ``AdamW`` for the embedding and the norms.

Tokens go through a table (``embedding``), the blocks of ``peri_blocks.py``, and
the same table again as the output's weight (``linear8``); ``cross_entropy_step`` gives the
loss and puts the gradient of the logits in their place.  The table's gradient is that of
the output first; ``embedding_backward`` adds the input's onto it.  The text is synthetic: each token
follows from the one before by a fixed rule, but for a tenth of them; a row's last token has no target.

    python examples/peri_lm.py --steps 100
"""

from __future__ import annotations

import argparse
import os
import sys
from typing import Dict, List, Tuple

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from peri_blocks import PeriBlocks, ops  # noqa: E402


class PeriLM(PeriBlocks):
    """PeriBlocks between a table and itself."""

    def __init__(self, vocab: int, d: int, hidden: int, blocks: int, kind: str = "rms"):
        super().__init__(d, hidden, blocks, kind)
        self.vocab = vocab
        self.table = (vocab, d)

    def parameters(self, device: torch.device, seed: int) -> Dict[str, torch.Tensor]:
        p = self.views(self.start(device, seed))
        gen = torch.Generator(device=device).manual_seed(seed + 1)
        p["table"] = torch.empty(self.table, device=device).normal_(0, self.d ** -0.5, generator=gen)
        return p

    def loss_and_gradients(self, p: Dict[str, torch.Tensor], g: Dict[str, torch.Tensor], tokens: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """The mean cross entropy; the gradients of ``p`` go into ``g`` (float32)."""
        scale = self.d ** 0.5
        out = self._weight("table", p["table"])
        n, kept = self.forward(p, ops.embedding(tokens, p["table"], scale=scale))
        loss, d = ops.cross_entropy_step(ops.linear8(n, out), targets, z_loss=1e-4, in_place=True)
        dn, _ = ops.linear8_backward(d, n, out, dw=g["table"])
        dx = self.backward(p, g, dn, kept)
        ops.embedding_backward(dx, tokens, self.vocab, scale=scale, dw=g["table"], accumulate=True)
        return loss


class Text:
    """Batches of (tokens, targets), [rows, length] each."""

    def __init__(self, vocab: int, rows: int, length: int, device: torch.device, seed: int):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.rows, self.length, self.device = vocab, rows, length, device

    def batch(self) -> Tuple[torch.Tensor, torch.Tensor]:
        draw = torch.randint(0, self.vocab, (self.rows, self.length), device=self.device, generator=self.gen)
        free = torch.rand((self.rows, self.length), device=self.device, generator=self.gen) < 0.1
        tokens = draw.clone()
        for t in range(1, self.length):
            tokens[:, t] = torch.where(free[:, t], draw[:, t], (3 * tokens[:, t - 1] + 1) % self.vocab)
        targets = torch.cat([tokens[:, 1:], torch.full((self.rows, 1), -1, device=self.device)], 1)
        return tokens, targets


def train(vocab: int = 512, d: int = 128, hidden: int = 256, blocks: int = 2, rows: int = 16, length: int = 64, steps: int = 100,
          lr: float = 0.02, say=print) -> List[float]:
    """The losses of the steps."""
    device = torch.device("cuda")
    net, text = PeriLM(vocab, d, hidden, blocks), Text(vocab, rows, length, device, 1)
    p = net.parameters(device, 0)
    g = {k: torch.empty_like(v) for k, v in p.items()}
    matrices = [k for k, v in p.items() if v.dim() == 2 and k != "table"]
    rest = [k for k in p if k not in matrices]
    muon = ops.Muon([p[k] for k in matrices], [g[k] for k in matrices], weight_decay=0.01)
    adamw = ops.AdamW([p[k] for k in rest], [g[k] for k in rest], betas=(0.9, 0.95))
    losses = []
    for step in range(steps):
        losses.append(net.loss_and_gradients(p, g, *text.batch()))
        muon.step(lr)
        adamw.step(0.1 * lr)
        if step % 20 == 0:
            say(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    muon.close()
    adamw.close()
    return torch.stack(losses).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("vocab", 512), ("d", 128), ("hidden", 256), ("blocks", 2), ("rows", 16), ("length", 64), ("steps", 100)):
        ap.add_argument(f"--{name}", type=int, default=value)
    losses = train(**vars(ap.parse_args()))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
