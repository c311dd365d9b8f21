"""Cross entropy (paper_2510_05361_amd.ops) at widths and numbers of rows that together reach
every kernel of it (test_lm_ops_instances.py), against the definition in 64 bits.  Bounds are those of
lm_oracle.cross_entropy: a running maximum that grows multiplies the sum so far by one more
exponential, whose error in its argument adds up to that of exp(x - m) itself, and by 3 U a turn of the loop, of which there are fewer
than a hundredth of the columns: within its cols / 64 + 28."""

import math

import pytest
import torch

import lm_oracle as oracle
from paper_2510_05361_amd import ops
from test_gpu_cross_entropy import DT, check, make

pytestmark = pytest.mark.gpu

# columns of rows that registers hold; the edges of each kernel
HELD = [512, 513, 1024, 1025, 1400, 2047, 2048, 2049, 3001, 4096, 4097, 8191, 16384, 16385, 32768, 32769, 57344, 57345, 60001, 65536, 131071]
# rows, columns of losses alone, as in evaluation
EVALUATION = [(511, 8193), (512, 8193), (515, 8193), (600, 32003), (1030, 12000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", HELD)
def test_rows_in_registers(cols, dtype):
    x, y = make(7, cols, dtype, none=0.0)
    low = torch.finfo(DT[dtype]).min
    y[1] = -1
    x[2, :cols - 1], y[2] = -math.inf, cols - 1  # one logit left, the last one
    x[3, 1:] = low
    x[4, cols // 2:], y[4] = -math.inf, 0
    x[5] = -math.inf                             # none left: NaN
    y[6] = cols                                  # not in the row: NaN
    for reduction, z in (("none", 0.0), ("none", 1e-3)):
        check(x, y, z, reduction, got=ops.cross_entropy(x.cuda(), y.cuda(), z_loss=z, reduction=reduction))
        loss, d = ops.cross_entropy_step(x.cuda(), y.cuda(), z_loss=z, reduction=reduction)
        check(x, y, z, reduction, got=loss, grad=d)
    assert loss[5:].isnan().all() and d[5:].isnan().all() and loss[1] == 0 and bool((d[1] == 0).all())
    loss, d = ops.cross_entropy_step(x[:5].cuda(), y[:5].cuda())
    check(x[:5], y[:5], got=loss, grad=d)


def check_sum(x, y, z, reduction, got):
    """As check; a sum of 2^128 (1 - 2^-25) and more, half a step above fp32's largest number 2^128 (1 - 2^-24), is rounded to
    infinity.  (Targets at a type's lowest value have losses of 3.4e38 each.)"""
    want, err, _, _ = oracle.cross_entropy(x.double(), y.long(), z)
    most = 2.0 ** 128 * (1 - 2.0 ** -25)
    if reduction == "sum" and float(want.sum() - err.sum()) >= most:
        assert got.item() == math.inf
    else:
        assert reduction == "mean" or float(want.sum() + err.sum()) < most
        check(x, y, z, reduction, got=got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", EVALUATION)
def test_losses_of_many_long_rows(rows, cols, dtype):
    x, y = make(rows, cols, dtype, none=0.05)
    low = torch.finfo(DT[dtype]).min
    at = torch.arange(rows)
    x[at % 7 == 1, :cols // 2] = -math.inf       # the first turns see nothing
    x[at % 7 == 2, cols // 3:] = -math.inf       # the last ones
    x[at % 7 == 3, :cols - 5] = low
    grow = at % 7 == 4                           # a maximum that grows at every turn
    x[grow] = (x[grow].float() + torch.linspace(-60, 60, cols)).to(DT[dtype])
    x[at % 7 == 5, 1:] = -math.inf               # one logit
    y[at % 7 == 5] = 0
    finite = x.float().gather(1, y.clamp(min=0)[:, None])[:, 0].isfinite() | (y < 0)
    for z in (0.0, 1e-4):
        check(x, y, z, "none", got=ops.cross_entropy(x.cuda(), y.cuda(), z_loss=z, reduction="none"))
        for reduction in ("sum", "mean"):
            check_sum(x[finite], y[finite], z, reduction, ops.cross_entropy(x[finite].cuda(), y[finite].cuda(), z_loss=z, reduction=reduction))
    # rows with nothing left, NaN, a target that is not there; the others as they are
    bad = x.clone()
    bad[10], bad[11, cols - 1], bad[12, 0] = -math.inf, math.nan, math.inf
    ids = y.clone()
    ids[10:13], ids[13], ids[14] = 3, cols, -1
    got = ops.cross_entropy(bad.cuda(), ids.cuda(), reduction="none")
    check(bad, ids, 0.0, "none", got=got)
    assert got[10:14].isnan().all() and got[14] == 0
    assert torch.equal(got[15:], ops.cross_entropy(x.cuda(), y.cuda(), reduction="none")[15:])


def test_losses_of_many_rows_between_gaps():
    """Rows apart, targets of 32 bits, in a graph, replayed with others."""
    x, y = make(520, 9001, "bf16", torch.int32)
    wide = torch.full((520, 9011), 90.0, dtype=torch.bfloat16, device="cuda")
    view, ids = wide[:, 5:9006], y.cuda()
    view.copy_(x)
    check(x, y, 0.0, "mean", got=ops.cross_entropy(view, ids))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = ops.cross_entropy(view, ids)
    for seed in (1, 2, 3):
        x, y = make(520, 9001, "bf16", torch.int32, seed)
        view.copy_(x)
        ids.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        check(x, y, 0.0, "mean", got=loss)
        assert torch.equal(loss, ops.cross_entropy(view, ids))
