"""8-bit blocks and their product (ops.quantize8, Weight8, product8, linear8)
against the definition in 64 bits.

Codes and scales have to be those of the definition, bit for bit.  Products,
with S = sum_k |a_k b_k| of the stored values and u = 2^-24:
- fp32 results: exact products summed in fp32, at most K/8 + 64 roundings in
  a row: (K/8 + 64) u S (the instructions may round each of four sums of 8);
- bf16 results: products more than 13 bits below the largest of their group
  of at most 16 may be dropped: 2^-9 S, and 2^-8 of the value for its rounding.
"""

import math

import pytest
import torch

import ops_oracle as oracle
from paper_2510_05361_amd import ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(shape, std=1.0, dtype="f32", seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(shape, device="cuda").normal_(0, std, generator=gen)
    # a few much larger columns, rows of different sizes
    if len(shape) == 2 and t.numel():
        t *= 1 + 20 * (torch.rand(shape[1], device="cuda", generator=gen) < 0.02)
        t *= torch.rand((shape[0], 1), device="cuda", generator=gen) * 4
    return t.to(DT[dtype])


def same_codes(q, codes, e):
    got = q.codes.double().cpu()
    assert got.shape == codes.shape
    assert torch.equal(got.isnan(), codes.isnan())
    assert torch.equal(got.nan_to_num(), codes.nan_to_num())
    s = q.scales.view(torch.uint8).cpu().long()
    assert torch.equal(s[:, :e.shape[1]], (e + 127).long())
    assert bool((s[:, e.shape[1]:] == 127).all())


SHAPES = [(1, 1), (1, 128), (3, 127), (5, 129), (128, 128), (130, 300), (257, 640), (64, 4096), (1000, 72)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_codes_and_scales(shape, dtype):
    x = rand(shape, dtype=dtype)
    along, across = oracle.rows8(x.cpu()), oracle.rows8(x.t().cpu())
    same_codes(ops.quantize8(x), *along)
    same_codes(ops.quantize8(x, rows=False, transposed=True), *across)
    both = ops.quantize8(x, transposed=True)
    same_codes(both[0], *along)
    same_codes(both[1], *across)
    w = ops.Weight8(x)
    codes, e = oracle.square8(x.cpu())
    same_codes(w.q, codes[:shape[0]], e)
    same_codes(w.qt, codes.t()[:shape[1]], e.t())
    assert torch.equal(w.q.dequantize().cpu().double(), oracle.values(codes[:shape[0]], e, 128)[:, :shape[1]])
    other = rand(shape, 3.0, dtype, seed=1)
    w.update(other)
    same_codes(w.q, oracle.square8(other.cpu())[0][:shape[0]], oracle.square8(other.cpu())[1])


def test_extreme_blocks():
    """Zeros, the smallest and largest fp32 values, powers of two and 448
    times them, infinities and NaN, ties."""
    x = torch.zeros((16, 256))
    x[1, 3] = 1.4e-45
    x[2, 200] = 3.4028234e38
    x[2, 5] = -1e30
    x[3, :128] = torch.exp2(torch.arange(-100, 28).float())
    x[4, 7], x[4, 140] = 448.0, 448.0 * (1 + 2.0 ** -23)
    x[5, 0], x[5, 1], x[5, 2], x[5, 3] = math.inf, -math.inf, math.nan, 5.0
    x[6, :] = math.nan
    x[7, :64] = torch.arange(64) + 0.5
    x[8, :] = 1e-40
    x[9, :128] = torch.linspace(-448, 448, 128)
    x[10, :128] = (torch.arange(128) - 64) * 2.0 ** -10
    x[10, 0] = 448.0
    same_codes(ops.quantize8(x.cuda()), *oracle.rows8(x))
    same_codes(ops.quantize8(x.cuda().t().contiguous(), rows=False, transposed=True), *oracle.rows8(x))
    codes, e = oracle.square8(x)
    same_codes(ops.Weight8(x.cuda()).q, codes[:16], e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_unaligned_inputs(dtype):
    wide = rand((70, 400), dtype=dtype)
    for view in (wide[:, 3:260], wide[::2, 1:], wide[5:, :131], wide.t()[1:], wide.view(-1)[1:27001].view(100, 270)):
        same_codes(ops.quantize8(view), *oracle.rows8(view.cpu()))
        same_codes(ops.quantize8(view, transposed=True)[1], *oracle.rows8(view.t().cpu()))


def stored(q):
    return q.dequantize().cpu().double()


def check_product(a, b, c, dtype, before=None):
    A, B = stored(a), stored(b)
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    if before is not None:
        want, size = want + before, size + before.abs()
    err = (A.shape[1] / 8 + 64) * U * size if dtype == "f32" else 2.0 ** -9 * size + 2.0 ** -8 * want.abs()
    diff = (c.cpu().double() - want).abs()
    assert bool((diff <= err + 1e-40).all()), float((diff / (err + 1e-40)).max())


PRODUCTS = [(1, 1, 1), (1, 200, 128), (2, 5, 300), (15, 129, 513), (16, 64, 64), (17, 1000, 256), (33, 300, 1152), (64, 128, 127),
            (65, 640, 520), (128, 128, 128), (129, 257, 384), (300, 77, 1000), (513, 520, 640), (1024, 768, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_products(m, n, k, weight, dtype):
    a = ops.quantize8(rand((m, k), seed=1))
    w = rand((n, k), 0.02, seed=2)
    b = ops.Weight8(w).q if weight else ops.quantize8(w)
    check_product(a, b, ops.product8(a, b, dtype=DT[dtype]), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(8, 64, 20000), (200, 130, 20001), (512, 1536, 8191), (2048, 2304, 768), (1999, 1025, 300), (256, 512, 16384),
                                   (4000, 2048, 128), (24, 8192, 2048), (40, 2048, 8192), (2000, 100, 5000)])
def test_larger_products(m, n, k, dtype):
    a, b = ops.quantize8(rand((m, k), seed=1)), ops.quantize8(rand((n, k), 0.02, seed=2))
    c = ops.product8(a, b, dtype=DT[dtype])
    check_product(a, b, c, dtype)
    assert torch.equal(c, ops.product8(a, b, dtype=DT[dtype])), "the order of the sums is fixed"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(4200, 2200, 384), (4097, 4100, 1), (2050, 8195, 700), (8200, 2048, 129)])
def test_products_of_many_tiles(m, n, k, dtype):
    """More than two 128 x 128 tiles a compute unit, ragged at both ends."""
    a, b = ops.quantize8(rand((m, k), seed=1)), ops.quantize8(rand((n, k), 0.02, seed=2))
    wide = torch.full((m, n + 3), 7.0, device="cuda").to(DT[dtype])
    c = wide[:, 1:1 + n]
    ops.product8(a, b, out=c)
    check_product(a, b, c, dtype)
    if dtype == "f32":
        keep = c.cpu().double()
        ops.product8(a, b, out=c, accumulate=True)
        check_product(a, b, c, dtype, keep)
    c[:] = 7.0
    assert bool((wide == 7.0).all())


@pytest.mark.parametrize("m,n,k", [(17, 33, 260), (30, 100, 1000), (49, 31, 4224), (64, 95, 130)])
def test_accumulate_to_few_rows(m, n, k):
    a, b = ops.quantize8(rand((m, k), seed=1)), ops.quantize8(rand((n, k), seed=2))
    c = torch.randn((m, n), device="cuda")
    keep = c.cpu().double()
    ops.product8(a, b, out=c, accumulate=True)
    check_product(a, b, c, "f32", keep)


@pytest.mark.parametrize("m,n,k", [(5, 7, 130), (8, 512, 4096), (300, 200, 520), (512, 520, 9000), (2100, 700, 128)])
def test_accumulate_and_strided_output(m, n, k):
    a, b = ops.quantize8(rand((m, k), seed=1)), ops.quantize8(rand((n, k), seed=2))
    wide = torch.randn((m, n + 9), device="cuda")
    keep = wide.clone()
    out = wide[:, 3:3 + n]
    ops.product8(a, b, out=out, accumulate=True)
    check_product(a, b, out, "f32", keep[:, 3:3 + n].cpu().double())
    assert torch.equal(wide[:, :3], keep[:, :3]) and torch.equal(wide[:, 3 + n:], keep[:, 3 + n:])
    for dtype in ("f32", "bf16"):
        wide = torch.full((m + 2, n + 9), 7.0, device="cuda").to(DT[dtype])
        ops.product8(a, b, out=wide[1:-1, 3:3 + n])
        check_product(a, b, wide[1:-1, 3:3 + n], dtype)
        wide[1:-1, 3:3 + n] = 7.0
        assert bool((wide == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [3, 200])
def test_non_finite_values_reach_their_rows_alone(m, dtype):
    x = rand((m, 500))
    x[1, 7], x[2, 450] = math.nan, math.inf
    a, b = ops.quantize8(x), ops.quantize8(rand((40, 500), seed=2))
    c = ops.product8(a, b, dtype=DT[dtype])
    rest = [i for i in range(m) if i not in (1, 2)]
    assert bool(c[rest].isfinite().all()) and bool(c[[1, 2]].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(4, 6, 260), (200, 140, 260)])
def test_scales_far_apart(m, n, k, dtype):
    """Blocks from 2^-60 to 2^60, and blocks of zeros."""
    a, b = rand((m, k), seed=1), rand((n, k), seed=2)
    a[:, :128] *= 2.0 ** -60
    a[1, 128:256] *= 2.0 ** 60
    b[:, 128:] *= 2.0 ** -50
    b[3] = 0
    a, b = ops.quantize8(a), ops.quantize8(b)
    check_product(a, b, ops.product8(a, b, dtype=DT[dtype]), dtype)


def test_empty_sizes():
    w = ops.Weight8(rand((40, 256)))
    assert ops.linear8(torch.empty((0, 256), device="cuda"), w).shape == (0, 40)
    dx, dw = ops.linear8_backward(torch.empty((0, 40), device="cuda"), torch.empty((0, 256), device="cuda"), w)
    assert dx.shape == (0, 256) and dw.shape == (40, 256) and bool((dw == 0).all())
    kept = torch.ones((40, 256), device="cuda")
    ops.linear8_backward(torch.empty((0, 40), device="cuda"), torch.empty((0, 256), device="cuda"), w, dw=kept, accumulate=True)
    assert bool((kept == 1).all())


@pytest.mark.parametrize("m", [1, 8, 77, 600])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_and_its_gradients(m, dtype):
    n, k = 200, 330
    x, dy, w = rand((m, k), dtype=dtype), rand((m, n), 1e-3, dtype, seed=3), rand((n, k), 0.02, seed=2)
    w8 = ops.Weight8(w)
    q = lambda t: oracle.values(*oracle.rows8(t.cpu()))[:, :t.shape[1]]  # noqa: E731
    wq = oracle.values(*oracle.square8(w.cpu()), 128)[:n, :k]

    def near(got, a, b):
        want, size = a @ b, a.abs() @ b.abs()
        err = (a.shape[1] / 8 + 64) * U * size if got.dtype == torch.float32 else 2.0 ** -9 * size + 2.0 ** -8 * want.abs()
        assert bool(((got.cpu().double() - want).abs() <= err + 1e-40).all())

    near(ops.linear8(x, w8), q(x), wq.t())
    dx, dw = ops.linear8_backward(dy, x, w8)
    assert dx.dtype == x.dtype and dw.dtype == torch.float32
    near(dx, q(dy), wq)
    near(dw, q(dy.t()), q(x.t()).t())
    # against the unrounded layer: four significant bits a side leave 2^-5 / sqrt(3) of every factor, and
    # the product is linear, so its difference along a direction is its value there
    exact = x.cpu().double() @ w.cpu().double().t()
    assert float((ops.linear8(x, w8).cpu().double() - exact).norm() / exact.norm()) < 0.06
    for got, want in ((dx, dy.cpu().double() @ w.cpu().double()), (dw, dy.cpu().double().t() @ x.cpu().double())):
        assert float((got.cpu().double() - want).norm() / want.norm()) < 0.06
    step = rand((m, k), dtype=dtype, seed=9)
    slope = float((dy.double() * (ops.linear8(step, w8).double() - ops.linear8(-step, w8).double()) / 2).sum())
    along = float((dx.double() * step.double()).sum())
    assert abs(slope - along) <= 0.06 * float(dx.double().norm() * step.double().norm()) 


def test_more_axes():
    w = ops.Weight8(rand((96, 256)))
    x = rand((30, 256), dtype="bf16")
    assert torch.equal(ops.linear8(x.view(2, 15, 256), w).view(30, 96), ops.linear8(x, w))


def test_codes_past_two_to_the_32():
    """A row-wise quantized matrix of more than 2^32 codes, and its product."""
    rows, k = (1 << 21) + 5, 2048
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1 << 20, (1 << 21) - 1, 1 << 21, rows - 1], device="cuda")
    x[some] = torch.randn((5, k), device="cuda").bfloat16()
    w = ops.Weight8(rand((130, k), 0.02))
    q, small = ops.quantize8(x), ops.quantize8(x[some])
    assert torch.equal(q.codes.view(torch.uint8)[some], small.codes.view(torch.uint8))
    y = ops.product8(q, w.q)
    assert torch.equal(y[some], ops.product8(ops.quantize8(x[:200].index_copy(0, torch.arange(5, device="cuda"), x[some])), w.q)[:5])
    assert int(y.abs().sum(1).nonzero().numel()) == 5


def test_side_stream_and_graph():
    x, dy = rand((300, 512), dtype="bf16"), rand((300, 384), dtype="bf16", seed=4)
    w = ops.Weight8(rand((384, 512), 0.02))
    call = lambda: (ops.linear8(x, w),) + ops.linear8_backward(dy, x, w)  # noqa: E731
    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        x.normal_()
        dy.normal_()
        torch.cuda.synchronize()
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    x = rand((4, 256))
    q, w = ops.quantize8(x), ops.Weight8(rand((8, 256)))
    for call in (lambda: ops.quantize8(x[0]), lambda: ops.quantize8(x, rows=False), lambda: ops.product8(q, w.q, accumulate=True),
                 lambda: ops.product8(q, w.q, out=torch.empty((4, 9), device="cuda")), lambda: ops.linear8(x[:, :128], w),
                 lambda: ops.linear8_backward(x, x, w), lambda: w.update(x), lambda: ops.product8(q, w.q, out=torch.empty((8, 4), device="cuda").t())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ops.quantize8(x.half())
    with pytest.raises(RuntimeError, match="columns"):
        ops.product8(q, ops.quantize8(rand((8, 130))))
    with pytest.raises(RuntimeError, match="accumulate"):
        ops.product8(q, w.q, out=torch.zeros((4, 8), device="cuda", dtype=torch.bfloat16), accumulate=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 3), (20, 5), (130, 259), (3000, 1030)])
def test_empty_contractions(m, n, dtype):
    """Sums over no columns are zero; with accumulate c stays as it is."""
    x, w = torch.empty((m, 0), dtype=DT[dtype], device="cuda"), torch.empty((n, 0), device="cuda")
    wide = torch.full((m + 2, n + 5), 7.0, device="cuda").to(DT[dtype])
    out = wide[1:-1, 3:3 + n]
    ops.product8(ops.quantize8(x), ops.quantize8(w), out=out)
    assert bool((out == 0).all())
    out[:] = 7.0
    assert bool((wide == 7.0).all())
    kept = torch.randn((m, n), device="cuda")
    before = kept.clone()
    ops.product8(ops.quantize8(x), ops.quantize8(w), out=kept, accumulate=True)
    assert torch.equal(kept, before)
    assert torch.equal(ops.linear8(x, ops.Weight8(w)), torch.zeros((m, n), dtype=DT[dtype], device="cuda"))
    assert ops.linear8(x.view(1, m, 0), ops.Weight8(w)).shape == (1, m, n)


@pytest.mark.parametrize("m", [3, 200])
def test_linear_of_no_outputs(m):
    w = ops.Weight8(torch.empty((0, 130), device="cuda"))
    x = rand((m, 130))
    assert ops.linear8(x, w).shape == (m, 0)
    dx, dw = ops.linear8_backward(torch.empty((m, 0), device="cuda"), x, w)
    assert dw.shape == (0, 130) and torch.equal(dx, torch.zeros((m, 130), device="cuda"))


def test_weight_dropped_with_a_call_in_flight_on_another_stream():
    """A weight quantized on one stream, used on a second one that waits for it, and
    dropped: its memory is not handed out before the call is done."""
    x, w = rand((300, 512), dtype="bf16"), rand((384, 512), 0.02)
    want = ops.linear8(x, ops.Weight8(w))
    held = ops.Weight8(w)
    ranges = [(m._buf.data_ptr(), m._buf.numel()) for m in (held.q, held.qt)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(240_000_000)  # a tenth of a second
        got = ops.linear8(x, held)
        got_dx = ops.linear8_backward(want, x, held)[0]
    del held
    fresh = [torch.full((size,), 127, dtype=torch.uint8, device="cuda") for _, size in ranges for _ in range(4)]
    busy = not side.query()
    for t in fresh:
        for at, size in ranges:
            assert t.data_ptr() + t.numel() <= at or at + size <= t.data_ptr()
    side.synchronize()
    assert busy, "the calls were to be in flight"
    assert torch.equal(got, want) and torch.equal(got_dx, ops.linear8_backward(want, x, ops.Weight8(w))[0])


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("w_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [5, 77])
def test_autograd(m, w_dtype, dtype, out):
    """Gradients through autograd are those of linear8_backward; the weight's goes
    to the tensor that it was made from."""
    x, w, dy = rand((m, 200), dtype=dtype), rand((90, 200), 0.02, w_dtype, seed=2), rand((m, 90), dtype=out, seed=3)
    common = DT[dtype] if dtype == out else torch.float32
    plain = ops.Weight8(w)
    want = ops.linear8_backward(dy.to(common), x.to(common), plain)
    for grads in ((True, True), (True, False), (False, True)):
        a, b = x.clone().requires_grad_(grads[0]), w.clone().requires_grad_(grads[1])
        held = ops.Weight8(b)
        y = ops.linear8(a.view(1, m, 200), held, dtype=DT[out])
        assert torch.equal(y[0], ops.linear8(x, plain, dtype=DT[out]))
        y.backward(dy[None])
        for t, g, needed in ((a, want[0], grads[0]), (b, want[1], grads[1])):
            assert (t.grad is not None) == needed
            assert not needed or t.grad.dtype == t.dtype and torch.equal(t.grad, g.to(t.dtype))
        with torch.no_grad():
            assert ops.linear8(a, held).grad_fn is None
    held.update(w)
    y = ops.linear8(a, held)
    held.update(w)
    with pytest.raises(RuntimeError, match="updated"):
        y.sum().backward()


def test_rows_past_one_row_of_workgroups():
    """More four rows by four blocks than go along x."""
    rows, k = (1 << 26) + 5, 8
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1 << 25, (1 << 26) - 5, (1 << 26) - 4, 1 << 26, rows - 1], device="cuda")
    x[some] = torch.randn((6, k), device="cuda").bfloat16()
    q, small = ops.quantize8(x), ops.quantize8(x[some])
    assert torch.equal(q.codes.view(torch.uint8)[some], small.codes.view(torch.uint8))
    assert torch.equal(q.scales.view(torch.uint8)[some], small.scales.view(torch.uint8))
    assert int(q.scales.view(torch.uint8)[:, 0].gt(1).sum()) == 6


@pytest.mark.parametrize("m", [8, 40])
def test_many_columns_and_few_rows(m):
    """More columns than workgroups go along x take."""
    n = (1 << 26) + 37
    a = ops.quantize8(rand((m, 100)))
    w = torch.zeros((n, 100), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1 << 24, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, n - 1], device="cuda")
    w[some] = torch.randn((7, 100), device="cuda").bfloat16()
    c = ops.product8(a, ops.quantize8(w))
    assert torch.equal(c[:, some], ops.product8(a, ops.quantize8(w[some])))
    assert int(c.abs().sum(0).nonzero().numel()) == 7


@pytest.mark.parametrize("outliers", [False, True])
@pytest.mark.parametrize("m,n,k", [(8, 8192, 2048), (48, 4096, 1000), (300, 520, 1024), (512, 1536, 4096), (2100, 2048, 700)])
def test_what_bf16_sums_leave_out(m, n, k, outliers):
    """bf16 results against the exact sums of the stored values, rounded.  Sums that
    are off by e of their norm, 0.8 e in the mean, cross a midpoint of bf16's steps
    (5.6e-3 of a value in the middle of its octave) in 0.8 e / 5.6e-3 of all cases
    and are then one step off: 5.6e-3 sqrt(0.8 e / 5.6e-3) of the norm.  For the
    stated e = 4e-5 that is 4.2e-4; twice that e is let pass, 6e-4.  fp32 results:
    k sums of like sizes, half a unit each at random."""
    gen = torch.Generator(device="cuda").manual_seed(k)
    x, w = torch.randn((m, k), device="cuda", generator=gen), torch.randn((n, k), device="cuda", generator=gen) * 0.02
    if outliers:
        x *= 1 + 20 * (torch.rand(k, device="cuda", generator=gen) < 0.02)
    a, b = ops.quantize8(x), ops.quantize8(w)
    want = stored(a) @ stored(b).t()
    got = ops.product8(a, b).cpu().double()
    assert float((got - want.bfloat16().double()).norm() / want.norm()) <= 6e-4
    assert float((ops.product8(a, b, dtype=torch.float32).cpu().double() - want).norm() / want.norm()) <= 4 * U * math.sqrt(k)


@pytest.mark.parametrize("rows,cols", [(0, 0), (0, 5), (0, 700), (5, 0), (200, 0)])
def test_matrices_without_elements_can_be_looked_at(rows, cols):
    x = torch.empty((rows, cols), device="cuda")
    up = lambda n, m: -(-n // m) * m  # noqa: E731
    for q, r, c, per in ((ops.quantize8(x), rows, cols, 1), (ops.quantize8(x, rows=False, transposed=True), cols, rows, 1),
                         (ops.Weight8(x).q, rows, cols, 128), (ops.Weight8(x).qt, cols, rows, 128)):
        assert q.codes.shape == (r, up(c, 128))
        assert q.scales.shape == (-(-r // per), up(c, 512) // 128)
        assert q.dequantize().shape == (r, c)


@pytest.mark.parametrize("m", [8, 48, 300])
def test_the_most_that_bf16_sums_leave_out(m):
    """One product of 2^16 in each eight, seven below 2^-13 of it, and as much of the
    other sign in the next block: what is left is the seven, of which each may be
    dropped.  At most 2^-10 of the sum of magnitudes, and the rounding."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    a = torch.randint(1, 3, (m, 512), device="cuda", generator=gen).float()
    b = torch.randint(1, 3, (64, 512), device="cuda", generator=gen).float()
    a[:, ::8], b[:, :256:8], b[:, 256::8] = 256, 256, -256
    qa, qb = ops.quantize8(a), ops.quantize8(b)
    want = a.cpu().double() @ b.cpu().double().t()
    size = a.cpu().double() @ b.abs().cpu().double().t()
    assert torch.equal(qa.dequantize(), a) and torch.equal(qb.dequantize(), b)
    got = ops.product8(qa, qb).cpu().double()
    assert bool(((got - want).abs() <= 2.0 ** -10 * size + 2.0 ** -8 * want.abs()).all())
    assert torch.equal(ops.product8(qa, qb, dtype=torch.float32).cpu().double(), want)
