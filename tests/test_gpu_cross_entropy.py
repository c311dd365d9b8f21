"""Cross entropy (paper_2510_05361_amd.ops) against the definition in 64 bits;
the bounds are those of lm_oracle.cross_entropy, with half a step of the result's
type for its rounding."""

import math

import pytest
import torch

import lm_oracle as oracle
from paper_2510_05361_amd import ops

pytestmark = pytest.mark.gpu

U = oracle.U
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(rows, cols, dtype="f32", ids=torch.int64, seed=0, none=0.2, std=3.0):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, cols), generator=gen) * std).to(DT[dtype])
    y = torch.randint(0, cols, (rows,), generator=gen, dtype=ids)
    y[torch.rand(rows, generator=gen) < none] = -1
    return x, y


def check(x, y, z=0.0, reduction="mean", scale=1.0, d_loss=None, got=None, grad=None):
    """got: the loss; grad: the gradient of the logits."""
    want, err, dx, derr = oracle.cross_entropy(x.double(), y.long(), z)
    n = max(1, int((y >= 0).sum()))
    over = n if reduction == "mean" else 1
    if got is not None:
        if reduction == "none":
            oracle.close(got, want, err + 1e-38)
        else:
            oracle.close(got, want.sum() / over, err.sum() / over + 2 * U * (want.sum() / over).abs() + 1e-38)
    if grad is not None:
        w = torch.full((x.shape[0], 1), scale / over, dtype=torch.float64) * (1.0 if d_loss is None else d_loss.double().view(-1, 1))
        want_d = dx * w
        oracle.close(grad, torch.where((y < 0)[:, None], torch.zeros_like(want_d), want_d),
                     derr * w.abs() + want_d.abs().nan_to_num() * (4 * U + oracle.half_step(x.dtype)) + 1e-38)


SIZES = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 1000), (70, 513), (4, 8192), (3, 8193), (9, 32003), (2, 50304), (2, 65537), (2, 131072), (1, 300001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, dtype):
    x, y = make(rows, cols, dtype)
    for reduction in ("none", "sum", "mean"):
        check(x, y, reduction=reduction, got=ops.cross_entropy(x.cuda(), y.cuda(), reduction=reduction))
        loss, d = ops.cross_entropy_step(x.cuda(), y.cuda(), reduction=reduction)
        check(x, y, reduction=reduction, got=loss, grad=d)
        assert d.dtype == x.dtype and loss.dtype == torch.float32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("z,scale,ids", [(1e-4, 1.0, torch.int32), (0.1, -2.5, torch.int64), (0.0, 0.125, torch.int32)])
def test_z_loss_scale_and_types_of_targets(z, scale, ids, dtype):
    x, y = make(33, 777, dtype, ids)
    loss, d = ops.cross_entropy_step(x.cuda(), y.cuda(), z_loss=z, scale=scale)
    check(x, y, z, scale=scale, got=loss, grad=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 9000, 140000])
def test_masked_columns_and_extreme_values(dtype, cols):
    """-inf, the type's lowest value, +inf and NaN in logits; targets that are masked."""
    x, y = make(12, cols, dtype, none=0.0)
    low = torch.finfo(DT[dtype]).min
    x[0, cols // 2:] = -math.inf          # half of a row masked
    y[0] = 3
    x[1, 1:] = -math.inf                  # one logit left
    y[1] = 0
    x[2] = -math.inf                      # none left: NaN
    x[3] = low                            # all equal, as low as can be
    x[4, ::2] = low
    y[4] = 1
    x[5, 5] = math.inf                    # NaN
    x[6, 6] = math.nan                    # NaN
    x[7, 9] = -math.inf                   # the target itself: an infinite loss
    y[7] = 9
    x[8] = 80.0                           # large, all equal
    x[9, 11] = 3e4                        # certain of another one
    x[10, 2], y[10] = 200.0, 2            # certain of the target
    x[11], y[11] = math.nan, -1           # nothing is asked of it
    losses = ops.cross_entropy(x.cuda(), y.cuda(), reduction="none")
    check(x, y, reduction="none", got=losses)
    assert losses[[2, 5, 6]].isnan().all() and losses[7].item() == math.inf and losses[11].item() == 0
    _, d = ops.cross_entropy_step(x.cuda(), y.cuda(), reduction="sum")
    check(x, y, reduction="sum", grad=d)
    assert bool((d[11] == 0).all()) and bool((d[0, cols // 2:] == 0).all())


def test_targets_outside_and_none_at_all():
    x, y = make(6, 50, none=0.0)
    y[2], y[4] = 50, 2 ** 40
    loss, d = ops.cross_entropy_step(x.cuda(), y.cuda(), reduction="none")
    check(x, y, reduction="none", got=loss, grad=d)
    assert loss[[2, 4]].isnan().all() and d[[2, 4]].isnan().all()
    y[:] = -100
    for reduction in ("mean", "sum"):
        loss, d = ops.cross_entropy_step(x.cuda(), y.cuda(), reduction=reduction)
        assert loss.item() == 0 and bool((d == 0).all())


def test_no_rows():
    x, y = torch.empty((0, 9), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    assert ops.cross_entropy(x, y).item() == 0 and ops.cross_entropy(x, y, reduction="none").shape == (0,)
    loss, d = ops.cross_entropy_step(x, y)
    assert loss.item() == 0 and d.shape == (0, 9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [100, 4097, 50304, 200000])
def test_strides_and_in_place(cols, dtype):
    x, y = make(7, cols, dtype)
    wide = torch.full((7, cols + 5), 7.0, dtype=DT[dtype], device="cuda")
    wide[:, 3:3 + cols] = x.cuda()
    view = wide[:, 3:3 + cols]
    loss, d = ops.cross_entropy_step(view, y.cuda())
    check(x, y, got=loss, grad=d)
    version = view._version
    loss, same = ops.cross_entropy_step(view, y.cuda(), in_place=True)
    assert same.data_ptr() == view.data_ptr() and view._version > version
    assert torch.equal(view, d) and bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + cols:] == 7).all())
    check(x, y, got=loss)


def test_one_row_and_views_that_cannot_be_written():
    x, y = make(1, 70, none=0.0)
    loss, d = ops.cross_entropy_step(x[0].cuda(), y[0].cuda())
    check(x, y, got=loss, grad=d[None])
    wide = torch.randn((70, 9), device="cuda")
    for bad in (wide.t(), x.cuda().expand(9, 70)):
        with pytest.raises(ValueError, match="in place"):
            ops.cross_entropy_step(bad, torch.zeros(9, dtype=torch.int64, device="cuda"), in_place=True)
    check(wide.t().cpu(), torch.zeros(9, dtype=torch.int64), grad=ops.cross_entropy_step(wide.t(), torch.zeros(9, dtype=torch.int64, device="cuda"))[1])


def test_gradients_that_are_broadcast():
    """The sum of single losses: one number for all of them, strides of zero."""
    x, y = make(9, 300)
    leaf = x.cuda().requires_grad_()
    ops.cross_entropy(leaf, y.cuda(), reduction="none").sum().backward()
    check(x, y, reduction="sum", grad=leaf.grad)


def test_batches_of_sequences():
    x, y = make(24, 300, "bf16")
    loss, d = ops.cross_entropy_step(x.view(4, 6, 300).cuda(), y.view(4, 6).cuda(), reduction="none")
    assert loss.shape == (4, 6) and d.shape == (4, 6, 300)
    check(x, y, reduction="none", got=loss.view(-1), grad=d.view(24, 300))
    # transposed targets and logits
    loss, d = ops.cross_entropy_step(x.view(4, 6, 300).cuda().transpose(0, 1), y.view(4, 6).cuda().t(), reduction="none")
    check(x, y, reduction="none", got=loss.t().reshape(-1), grad=d.transpose(0, 1).reshape(24, 300))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_autograd(reduction, dtype):
    x, y = make(20, 640, dtype)
    leaf = x.cuda().requires_grad_()
    loss = ops.cross_entropy(leaf, y.cuda(), z_loss=1e-3, reduction=reduction)
    up = torch.linspace(-1, 2, 20) if reduction == "none" else torch.tensor(0.75)
    loss.backward(up.cuda())
    check(x, y, 1e-3, reduction, d_loss=up, got=loss.detach(), grad=leaf.grad)


def test_gradient_against_differences():
    x, y = make(4, 60, std=1.0)
    _, d = ops.cross_entropy_step(x.cuda(), y.cuda(), z_loss=0.01)
    h = 2.0 ** -7  # losses off by 2^-22, differences of h^2: 2^-14 and less
    for j in (0, 17, int(y[y >= 0][0])):
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        each = [ops.cross_entropy(t.cuda(), y.cuda(), z_loss=0.01, reduction="sum").item() for t in (up, down)]
        assert abs((each[0] - each[1]) / (2 * h) / int((y >= 0).sum()) - d[:, j].sum().item()) < 2e-4


def test_same_results_again_and_in_a_graph():
    """Deterministic, and the same replayed, with eager work between replays."""
    x, y = (t.cuda() for t in make(300, 5000, "bf16"))
    first = ops.cross_entropy_step(x, y)
    assert all(torch.equal(a, b) for a, b in zip(first, ops.cross_entropy_step(x, y)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.cross_entropy_step(x, y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.cross_entropy_step(x, y)
    for seed in (1, 2, 3):
        nx, ny = make(300, 5000, "bf16", seed=seed)
        x.copy_(nx)
        y.copy_(ny)
        graph.replay()
        torch.cuda.synchronize()
        eager = ops.cross_entropy_step(x, y)
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_a_row_past_32_bits_of_elements():
    """Offsets beyond 2^31 elements: the last rows of 5 GB of logits."""
    rows, cols = 45000, 50304
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.normal_(0, 2, generator=torch.Generator(device="cuda").manual_seed(0))
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    y[-3:] = torch.tensor([5, 50303, 0], dtype=torch.int32)
    tail, ty = x[-4:].cpu(), y[-4:].cpu()
    loss, d = ops.cross_entropy_step(x, y, in_place=True)
    check(tail, ty, got=loss, grad=d[-4:])
    assert bool((d[0] == 0).all()) and bool((d[rows // 2] == 0).all())
