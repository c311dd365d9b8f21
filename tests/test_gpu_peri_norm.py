"""The boundary of a Peri-LN block (ops.peri_norm, ops.peri_norm_backward)
against the definition in 64 bits and its derivative.

Tolerances, with u = 2^-24 and rows of D elements summed by a tree of depth
below 24 after at most 32 sequential sums per thread: a statistic (a mean of
squares, a mean) is off by at most 40u of the mean of its magnitudes, which
the fp32 sums of LayerNorm's centring add |mean| 40u to every centred value.
A row's outputs are then off by 64u of the sum of the magnitudes of their
terms (below: `terms`, with |z - mean| + |mean| in the place of |z - mean|);
sums over T rows by (T + 64) u at most of the sum of magnitudes; bf16 storage
adds 2^-8 of the value (eight significant bits).
"""

import math

import pytest
import torch

import ops_oracle as oracle
from paper_2510_05361_amd import ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(t, d, stream="f32", branch="f32", w="f32", gate=None, seed=0, mean=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype, mu=0.0):
        return torch.empty(shape, device="cuda").normal_(mu, std, generator=gen).to(DT[dtype])

    s = {"x": normal((t, d), 1.0, stream, mean), "f": normal((t, d), 0.5, branch, mean), "w_post": normal(d, 0.2, w, 1.0),
         "w_pre": normal(d, 0.2, w, 1.0), "d_out": normal((t, d), 1.0, stream), "dn": normal((t, d), 1.0, branch)}
    s["gate"] = normal((-(-t // gate), d), 0.5, w, 0.5) if gate else None
    return s


def d64(t):
    return None if t is None else t.detach().cpu().double()


def near(got, want, terms, bf16, what, factor=64):
    err = factor * U * terms + (2.0 ** -8 * want.abs() * (1 + 1e-5) if bf16 else 0.0) + 1e-40
    diff = (got.cpu().double() - want).abs()
    assert bool((diff <= err).all()), f"{what}: {float((diff / err).max())} of the bound"


def magnitudes(z, w, layer):
    """Bound of the magnitudes that go into norm(z) w, elementwise."""
    mean = z.mean(-1, keepdim=True) if layer else torch.zeros(())
    r = ((z - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()
    return ((z - mean).abs() + mean.abs()) * r * w.abs() * (1 + (mean.abs() * r) ** 2)


def check_forward(s, kind, rows_per_gate, scale, **layout):
    layer = kind == "layer"
    a = {k: layout.get(k, s[k]) for k in ("x", "f")}
    out, n = ops.peri_norm(a["x"], a["f"], s["w_post"] if s["f"] is not None else None, s["w_pre"], gate=s["gate"],
                           rows_per_gate=rows_per_gate, scale=scale, eps=EPS, kind=kind)
    r = {k: d64(s[k]) for k in ("x", "f", "w_post", "w_pre", "gate")}
    per = rows_per_gate or max(1, r["x"].shape[0])
    want, want_n = oracle.peri_norm(r["x"], r["f"], r["w_post"], r["w_pre"], r["gate"], per, scale, EPS, layer)
    terms = r["x"].abs()
    if s["f"] is not None:
        g = 1.0 if r["gate"] is None else r["gate"][torch.arange(r["x"].shape[0]) // per].abs()
        terms = terms + abs(scale) * g * magnitudes(r["f"], r["w_post"], layer)
        near(out, want, terms, s["x"].dtype == torch.bfloat16, "x'")
    else:
        assert out.data_ptr() == a["x"].data_ptr()
    if s["w_pre"] is not None:
        mean = want.mean(-1, keepdim=True) if layer else torch.zeros(())
        rr = ((want - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()
        # x' is off by 64u terms; a statistic by the mean of what its elements are off by
        each = (terms + terms.square().mean(-1, keepdim=True).sqrt()) * rr * (1 + (want - mean).abs() * rr) * r["w_pre"].abs()
        near(n, want_n, each * (1 + (mean.abs() * rr) ** 2), n.dtype == torch.bfloat16, "n", 128)
    else:
        assert n is None


def check_backward(s, kind, rows_per_gate, scale, **layout):
    layer = kind == "layer"
    a = {k: layout.get(k, s[k]) for k in ("x", "f", "d_out", "dn")}
    got = ops.peri_norm_backward(a["d_out"], a["dn"], a["x"], a["f"], s["w_post"] if s["f"] is not None else None, s["w_pre"],
                                 gate=s["gate"], rows_per_gate=rows_per_gate, scale=scale, eps=EPS, kind=kind)
    got = dict(zip(("x", "f", "w_post", "w_pre", "gate"), got))
    r = {k: d64(s[k]) for k in ("x", "f", "w_post", "w_pre", "gate", "d_out", "dn")}
    t = r["x"].shape[0]
    per = rows_per_gate or max(1, t)
    want = oracle.peri_norm_backward(r["d_out"], r["dn"], r["x"], r["f"], r["w_post"], r["w_pre"], r["gate"], per, scale, EPS, layer)
    for k in ("f", "w_post", "w_pre", "gate"):
        assert (got[k] is None) == (k not in want), k

    def through(y, z):  # magnitudes of the gradient through norm(z)
        mean = z.mean(-1, keepdim=True) if layer else torch.zeros(())
        rr = ((z - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()
        zh = ((z - mean).abs() + mean.abs()) * rr
        lost = 1 + (mean.abs() * rr) ** 2
        return rr * lost * (y + y.mean(-1, keepdim=True) + zh * (y * zh).mean(-1, keepdim=True)), zh * lost

    dmag = torch.zeros_like(r["x"]) if r["d_out"] is None else r["d_out"].abs()
    if r["w_pre"] is not None:
        y = torch.zeros_like(r["x"]) if r["dn"] is None else r["dn"].abs()
        more, zh = through(y * r["w_pre"].abs(), r["x"])
        dmag = dmag + 2 * more
        near(got["w_pre"], want["w_pre"], (y * zh).sum(0), False, "w_pre", t + 128)
    near(got["x"], want["x"], dmag, got["x"].dtype == torch.bfloat16, "dx")
    if r["f"] is not None:
        g = torch.ones(()) if r["gate"] is None else r["gate"][torch.arange(t) // per].abs()
        dh = abs(scale) * g * dmag
        more, fh = through(dh * r["w_post"].abs(), r["f"])
        near(got["f"], want["f"], 4 * more, got["f"].dtype == torch.bfloat16, "df")
        near(got["w_post"], want["w_post"], (dh * fh).sum(0), False, "w_post", t + 192)
        if r["gate"] is not None:
            each = oracle.pad_to((dmag * fh * r["w_post"].abs() * abs(scale)).t().contiguous(), per).view(-1, r["gate"].shape[0], per).sum(-1).t()
            near(got["gate"], want["gate"], each, False, "gate", per + 192)


WIDTHS = [1, 7, 8, 9, 64, 511, 512, 513, 768, 1024, 1030, 2048, 2049, 4096, 4104, 8191, 8192]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, kind):
    s = inputs(5, d, gate=2)
    check_forward(s, kind, 2, 0.7)
    check_backward(s, kind, 2, 0.7)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("stream,branch,w", [("bf16", "bf16", "bf16"), ("bf16", "bf16", "f32"), ("f32", "bf16", "f32"),
                                             ("f32", "f32", "bf16")])
@pytest.mark.parametrize("d", [72, 768, 2050, 5000])
def test_types(stream, branch, w, kind, d):
    s = inputs(9, d, stream, branch, w, gate=9)
    check_forward(s, kind, 0, -1.5)
    check_backward(s, kind, 0, -1.5)


@pytest.mark.parametrize("stream,branch,kind", [("bf16", "bf16", "rms"), ("f32", "bf16", "layer"), ("f32", "f32", "rms")])
@pytest.mark.parametrize("t,d", [(1500, 1000), (1100, 1021), (700, 2048), (515, 2050), (300, 4096), (260, 4100), (200, 5003), (170, 8192), (90, 8192)])
def test_widths_of_many_rows(t, d, stream, branch, kind):
    s = inputs(t, d, stream, branch, gate=97)
    check_forward(s, kind, 97, 0.7)
    check_backward(s, kind, 97, 0.7)


@pytest.mark.parametrize("t", [1, 2, 3, 31, 600, 4099])
@pytest.mark.parametrize("gate", [None, 1, 2, 7, 300, 5000])
@pytest.mark.parametrize("d", [96, 1000])
def test_rows_and_gates(t, gate, d):
    s = inputs(t, d, gate=gate)
    check_forward(s, "rms", gate or 0, 0.5)
    check_backward(s, "rms", gate or 0, 0.5)


@pytest.mark.parametrize("t,d,gate", [(4452, 300, 5), (4452, 300, 6), (4452, 300, 7), (2500, 1500, 4), (2500, 1500, 8), (2500, 1500, 9), (600, 2056, 3),
                                      (600, 4100, 2), (600, 4100, 4), (9000, 64, 18), (9000, 64, 11), (3000, 1021, 5), (2100, 900, 64)])
def test_gates_of_a_few_rows(t, d, gate):
    """Gates that a workgroup has whole, several or one, and those it has not."""
    s = inputs(t, d, "f32", "bf16", gate=gate)
    check_backward(s, "layer", gate, 0.5)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("drop", [("f",), ("w_pre",), ("d_out",), ("dn",), ("f", "d_out"), ("w_pre", "gate"), ("gate",)])
@pytest.mark.parametrize("d", [200, 2500])
def test_missing_parts(drop, kind, d):
    s = inputs(21, d, gate=4)
    for k in drop + (("gate",) if "f" in drop else ()) + (("dn",) if "w_pre" in drop else ()):
        s[k] = None
    per = 4 if s["gate"] is not None else 0
    check_forward(s, kind, per, 0.5)
    check_backward(s, kind, per, 0.5)


@pytest.mark.parametrize("d", [33, 1000])
def test_strides(d):
    """Rows of wider buffers, at odd offsets; transposed inputs are copied."""
    s = inputs(12, d)
    views = {}
    for k in ("x", "f", "d_out", "dn"):
        wide = torch.full((12, d + 13), math.nan, device="cuda", dtype=s[k].dtype)
        views[k] = wide[:, 5:5 + d]
        views[k].copy_(s[k])
    check_forward(s, "rms", 0, 0.5, **{k: views[k] for k in ("x", "f")})
    check_backward(s, "rms", 0, 0.5, **views)
    turned = {k: s[k].t().contiguous().t() for k in views}
    check_forward(s, "layer", 0, 0.5, **{k: turned[k] for k in ("x", "f")})
    check_backward(s, "layer", 0, 0.5, **turned)


def test_more_axes_and_no_rows():
    s = inputs(24, 40)
    flat = ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"])
    deep = ops.peri_norm(s["x"].view(2, 3, 4, 40), s["f"].view(2, 3, 4, 40), s["w_post"], s["w_pre"])
    assert all(torch.equal(a, b.view(24, 40)) for a, b in zip(flat, deep))
    e = s["x"][:0]
    out, n = ops.peri_norm(e, e, s["w_post"], s["w_pre"])
    assert out.shape == n.shape == (0, 40)
    got = ops.peri_norm_backward(e, e, e, e, s["w_post"], s["w_pre"], gate=s["w_post"][None])
    assert got[0].shape == (0, 40)
    assert all(bool((g == 0).all()) and g.numel() == 40 for g in got[2:])


@pytest.mark.parametrize("d", [100, 3000])
def test_large_mean_constant_and_zero_rows(d):
    """LayerNorm of rows with a mean of 300 deviations, of constant rows and
    of zeros; RMS of zeros."""
    s = inputs(6, d, mean=300.0)
    check_forward(s, "layer", 0, 0.5)
    check_backward(s, "layer", 0, 0.5)
    s = inputs(6, d)
    s["f"][2], s["f"][3], s["x"][3] = 2.0, 0.0, 0.0
    for kind in ("rms", "layer"):
        check_forward(s, kind, 0, 0.5)
        check_backward(s, kind, 0, 0.5)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [24, 100])
def test_rows_whose_squares_vanish(d, kind):
    """eps = 0 and rows of 1e-20, whose mean square lies below the smallest
    normal number (three decades above the smallest there is: 2^-149 more in
    every sum of squares, d of them, a relative 2^-14 of the root at most)."""
    s = inputs(6, d, gate=None)
    s["x"] *= 2.0 ** -66
    s["f"] *= 2.0 ** -64
    x, f, w, v = (s[k].cpu().double() for k in ("x", "f", "w_post", "w_pre"))
    out, n = ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"], eps=0.0, kind=kind, scale=2.0 ** -66)
    want, want_n = oracle.peri_norm(x, f, w, v, None, 6, 2.0 ** -66, 0.0, kind == "layer")
    assert bool(((out.cpu().double() - want).abs() <= 2.0 ** -13 * (want.abs() + x.abs())).all())
    assert bool(((n.cpu().double() - want_n).abs() <= 2.0 ** -10 * want_n.abs().amax()).all())


@pytest.mark.parametrize("d", [100, 3000])
def test_non_finite_rows_stay_alone(d):
    s = inputs(8, d)
    clean = ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"])
    s["f"][2, 7], s["x"][5, 9] = math.inf, math.nan
    out, n = ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"])
    keep = [0, 1, 3, 4, 6, 7]
    assert torch.equal(out[keep], clean[0][keep]) and torch.equal(n[keep], clean[1][keep])
    assert not bool(n[[2, 5]].isfinite().any(-1).all())
    dx, df, *_ = ops.peri_norm_backward(s["d_out"], s["dn"], out, s["f"], s["w_post"], s["w_pre"])
    assert bool(dx[keep].isfinite().all()) and bool(df[keep].isfinite().all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradient_against_differences(kind):
    """<gradient, direction> against the central difference of the loss
    <a, x'> + <b, n> along it, every input at once.  With steps of 2^-6 the
    difference is off by the loss's third derivative, about 2^-12 of the
    gradient's size here, and by rounding, u 2^6 of the loss's terms."""
    t, d, per = 40, 96, 7
    s = inputs(t, d, gate=per)
    names = ("x", "f", "w_post", "w_pre", "gate")
    a, b = s["d_out"], s["dn"]

    def forward(k):
        v = {n: s[n] + k * dirs[n] for n in names}
        return ops.peri_norm(v["x"], v["f"], v["w_post"], v["w_pre"], gate=v["gate"], rows_per_gate=per, scale=0.5, eps=EPS, kind=kind)

    gen = torch.Generator(device="cuda").manual_seed(3)
    for name in names:
        dirs = {n: torch.randn(s[n].shape, device="cuda", generator=gen) if n == name else torch.zeros_like(s[n]) for n in names}
        h = 2.0 ** -6
        diff = sum(float((w.double() * (p.double() - m.double())).sum()) for w, p, m in zip((a, b), forward(h), forward(-h))) / (2 * h)
        out, _ = forward(0.0)
        got = dict(zip(names, ops.peri_norm_backward(a, b, out, s["f"], s["w_post"], s["w_pre"], gate=s["gate"], rows_per_gate=per,
                                                     scale=0.5, eps=EPS, kind=kind)))
        want = float((got[name].double() * dirs[name].double()).sum())
        size = float(got[name].double().norm() * dirs[name].double().norm()) / math.sqrt(dirs[name].numel())
        assert abs(diff - want) <= 2e-2 * size, (name, diff, want, size)


def test_rows_past_two_to_the_32_elements():
    t, d = (1 << 20) + 3, 4096
    x = torch.zeros((t, d), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1 << 19, (1 << 20) - 1, 1 << 20, t - 1], device="cuda")
    x[some] = torch.randn((5, d), device="cuda").bfloat16()
    w = torch.ones(d, device="cuda")
    small, big = ops.peri_norm(x[some], x[some], w, w), ops.peri_norm(x, x, w, w)
    assert all(torch.equal(b[some], a) for a, b in zip(small, big))
    del big
    s_small = ops.peri_norm_backward(x[some], x[some], x[some], x[some], w, w)
    s_big = ops.peri_norm_backward(x, x, x, x, w, w)
    assert torch.equal(s_big[0][some], s_small[0]) and torch.equal(s_big[1][some], s_small[1])
    for a, b in zip(s_small[2:4], s_big[2:4]):
        assert bool(((a - b).abs() <= 16 * U * a.abs() + 1e-4).all())


def test_determinism_side_stream_and_graph():
    s = inputs(3000, 768, "bf16", "bf16", gate=500)
    call = lambda: ops.peri_norm_backward(s["d_out"], s["dn"], s["x"], s["f"], s["w_post"], s["w_pre"], gate=s["gate"], rows_per_gate=500)  # noqa: E731
    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call() + ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"])
    for _ in range(3):
        s["dn"].normal_()
        s["f"].normal_()
        torch.cuda.synchronize()
        graph.replay()
        want = call() + ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    s = inputs(4, 64)
    x, f, w = s["x"], s["f"], s["w_post"]
    for call in (lambda: ops.peri_norm(x, f[:2], w, w), lambda: ops.peri_norm(x, f, None, w), lambda: ops.peri_norm(x, None, None, None),
                 lambda: ops.peri_norm(x, f, w[:8], w), lambda: ops.peri_norm(x, f, w, w.bfloat16()),
                 lambda: ops.peri_norm(x, f, w, w, kind="batch"), lambda: ops.peri_norm(x, f, w, w, gate=w[None], rows_per_gate=2),
                 lambda: ops.peri_norm(x, f, w, w.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.peri_norm(x.half(), f, w, w), lambda: ops.peri_norm(x, f.half(), w, w),
                 lambda: ops.peri_norm_backward(x.bfloat16(), f, x, f, w, w)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ops.peri_norm(x.bfloat16(), f, w, w), lambda: ops.peri_norm(x, f, w, w, eps=-1.0),
                 lambda: ops.peri_norm(torch.zeros(2, 8193, device="cuda"), None, None, torch.ones(8193, device="cuda"))):
        with pytest.raises(RuntimeError):
            call()


@pytest.mark.parametrize("per", [0, 3])
def test_gradients_of_no_rows_at_the_c_entry(per):
    """Sums over no rows are zero."""
    from paper_2510_05361_amd import mtdao_ops as c_ops
    d = 72
    w = torch.ones(d, device="cuda")
    sums = torch.full((2, d), 7.0, device="cuda")
    a = c_ops.PeriNormArgs()
    a.rows, a.d, a.eps, a.scale, a.rows_per_gate = 0, d, EPS, 0.5, per
    a.ld_x = a.ld_f = a.ld_d_out = a.ld_dn = d
    a.f = a.w_post = a.w_pre = w.data_ptr()
    a.d_w_post, a.d_w_pre = sums[0].data_ptr(), sums[1].data_ptr()
    if per:
        a.gate, a.d_gate = w.data_ptr(), w.data_ptr()
    assert c_ops.mtdao_peri_norm_backward_workspace_bytes(a) == 0
    c_ops.mtdao_peri_norm_backward(a, None, 0, torch.cuda.current_stream().cuda_stream)
    assert bool((sums == 0).all()) and bool((w == 1).all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("t,d,gate", [(1, 24, None), (6, 24, None), (7, 100, 2), (3, 2048, None), (11, 1000, 3), (1030, 700, 5), (5, 5000, 2)])
@pytest.mark.parametrize("drop", [(), ("w_pre", "dn"), ("f", "gate"), ("d_out",)], ids=str)
def test_gradients_without_eps(t, d, gate, kind, drop, monkeypatch):
    """eps = 0, with rows that leave some of a workgroup's shares empty: finite
    gradients, as the definition has them."""
    monkeypatch.setitem(globals(), "EPS", 0.0)
    s = inputs(t, d, gate=gate)
    for k in drop:
        s[k] = None
    check_backward(s, kind, gate if gate and s["gate"] is not None else 0, 0.5)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [100, 2048])
def test_gradient_of_an_output_that_is_not_there(d, kind):
    """Without w_pre there is no n: dn has no part in the gradients, whatever it holds."""
    s = inputs(9, d)
    want = ops.peri_norm_backward(s["d_out"], None, s["x"], s["f"], s["w_post"], None, kind=kind)
    got = ops.peri_norm_backward(s["d_out"], torch.full_like(s["dn"], math.nan), s["x"], s["f"], s["w_post"], None, kind=kind)
    for a, b in zip(got, want):
        assert a is b is None or torch.equal(a, b)


@pytest.mark.parametrize("per", [41, 2 ** 31, 2 ** 63 - 1, 2 ** 70])
def test_one_gate_for_more_rows_than_there_are(per):
    s = inputs(40, 96, gate=40)
    a, b = ((ops.peri_norm(s["x"], s["f"], s["w_post"], s["w_pre"], gate=s["gate"], rows_per_gate=n) +
             ops.peri_norm_backward(s["d_out"], s["dn"], s["x"], s["f"], s["w_post"], s["w_pre"], gate=s["gate"], rows_per_gate=n))
            for n in (per, 40))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("drop", [(), ("f", "w_post", "gate"), ("w_pre",), ("gate",)], ids=str)
@pytest.mark.parametrize("stream,branch,w", [("f32", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32")])
def test_autograd(stream, branch, w, drop, kind):
    """Gradients through autograd are those of peri_norm_backward, in their tensors'
    types; of either output alone too.  A part without requires_grad takes none."""
    s = inputs(30, 200, stream, branch, w, gate=7)
    names = [k for k in ("x", "f", "w_post", "w_pre", "gate") if k not in drop]
    leaves = {k: s[k].clone().requires_grad_() if k in names else None for k in ("x", "f", "w_post", "w_pre", "gate")}
    how = dict(rows_per_gate=0 if leaves["gate"] is None else 7, scale=0.5, kind=kind)

    def forward(v):
        return ops.peri_norm(v["x"], v["f"], v["w_post"], v["w_pre"], gate=v["gate"], branch_dtype=DT[branch], **how)

    with torch.no_grad():
        plain = forward(leaves)
    assert not any(t is not None and t.grad_fn is not None for t in plain)
    for given in ((True, True), (True, False), (False, True)):
        out, n = forward(leaves)
        assert torch.equal(out, plain[0]) and (n is plain[1] is None or torch.equal(n, plain[1]))
        d_out, dn = (s[k] if use else None for k, use in zip(("d_out", "dn"), given))
        dn = dn if n is not None else None
        pairs = [(t, g) for t, g in ((out, d_out), (n, dn)) if g is not None]
        if not pairs or leaves["f"] is None and dn is None:
            continue
        got = torch.autograd.grad([t for t, _ in pairs], [leaves[k] for k in names], [g for _, g in pairs], allow_unused=True)
        want = dict(zip(("x", "f", "w_post", "w_pre", "gate"), ops.peri_norm_backward(
            d_out if leaves["f"] is not None else None, dn, plain[0], s["f"] if leaves["f"] is not None else None,
            *(s[k] if leaves[k] is not None else None for k in ("w_post", "w_pre")), gate=s["gate"] if leaves["gate"] is not None else None, **how)))
        if leaves["f"] is None and d_out is not None:
            want["x"] = want["x"] + d_out  # x' is x itself
        for k, g in zip(names, got):
            assert g.dtype == leaves[k].dtype and torch.equal(g, want[k].to(g.dtype)), (k, given)
    if "f" in names:
        some = {k: t if t is None or k == "f" else t.detach() for k, t in leaves.items()}
        out, _ = forward(some)
        out.float().sum().backward()
        assert leaves["f"].grad is not None and leaves["x"].grad is None


def test_rows_past_one_row_of_workgroups():
    """Four rows a workgroup and 2^21 workgroups along x: many narrow rows."""
    t, d = (1 << 24) + 5, 8
    x = torch.zeros((t, d), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1 << 23, (1 << 23) + 3, (1 << 24) - 1, 1 << 24, t - 1], device="cuda")
    x[some] = torch.randn((6, d), device="cuda").bfloat16()
    w = torch.ones(d, device="cuda")
    small, big = ops.peri_norm(x[some], x[some], w, w), ops.peri_norm(x, x, w, w)
    for a, b in zip(small, big):
        assert torch.equal(b[some], a) and int(b.abs().sum(1).nonzero().numel()) == 6
