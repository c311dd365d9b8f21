"""What the operators of include/mtdao_ops.h launch (CPU: launches are taken
down, nothing runs; addresses are numbers)."""

import pytest

import launch_recorder


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    shim = launch_recorder.build(str(tmp_path_factory.mktemp("shim")))
    return lambda body: launch_recorder.run(shim, body)


def names(launches):
    return [name for name, *_ in launches]


# ------------------------------------------------------------ 8-bit product


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("m,n", [(1, 5), (40, 5), (600, 700), (40000, 4000)])
def test_empty_contractions_read_no_matrix(run, m, n, dtype):
    """Products over no columns, whose codes and scales may be NULL: zeros, or
    nothing where c is added to."""
    launches, _ = run(f"""
        B = 1 << 40
        empty = lambda rows, scale_rows=1: c.Matrix8(None, None, rows, 0, 128, 4 * -(-rows // scale_rows), scale_rows)
        c.mtdao_product8(empty({m}), empty({n}), B, {dtype}, {n}, False, None, 0, None)
        c.mtdao_linear8(B, {dtype}, {m}, 0, empty({n}, 128), B << 1, {dtype}, {n}, None, 0, None)
        c.mtdao_product8(empty({m}), empty({n}), B, 0, {n}, True, None, 0, None)
    """)
    assert names(launches) == ["k_product8_zero"] * 2


@pytest.mark.parametrize("tokens,outputs,inputs", [(0, 40, 256), (0, 700, 3000), (30, 0, 256), (3, 0, 40)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_linear_gradients_of_nothing(run, tokens, outputs, inputs, accumulate):
    """No tokens: dw = 0 (or as it was).  No outputs: dx = 0.  The workspace holds
    no scales of matrices without columns."""
    launches, _ = run(f"""
        B = 1 << 40
        t, n, k = {tokens}, {outputs}, {inputs}
        wt = c.Matrix8(B, B + (1 << 30), k, n, max(1, -(-n // 128)) * 128, 4 * -(-k // 128), 128)
        need = c.mtdao_linear8_workspace_bytes(t, n, k)[1]
        c.mtdao_linear8_backward(B << 1, B << 2, 0, t, n, k, wt, B << 3, k, B << 4, k, {accumulate}, B << 5, need, None)
    """)
    assert names(launches) == ([] if tokens == 0 and accumulate else ["k_product8_zero"])


def test_products_with_a_contraction(run):
    """... launch what they did."""
    launches, _ = run("""
        B = 1 << 40
        def matrix(rows, cols, at, scale_rows=1):
            return c.Matrix8(at, at + (1 << 36), rows, cols, -(-cols // 128) * 128, 4 * -(-rows // scale_rows), scale_rows)
        for m, n, k in ((8, 512, 256), (64, 512, 1), (300, 512, 1), (2000, 512, 128), (8192, 8192, 128), (1536, 512, 8191)):
            need = c.mtdao_product8_workspace_bytes(m, n, k)
            c.mtdao_product8(matrix(m, k, B), matrix(n, k, B + (1 << 38)), B << 2, 0, n, False, B << 3, need, None)
    """)
    assert names(launches) == ["k_product8_few"] * 2 + ["k_product8_tiles"] * 4 + ["k_product8_join"]


# -------------------------------------------------------- Peri-LN boundary

PERI = """
        B = 1 << 40
        def peri(rows, d, per=0, drop=(), **kw):
            a = c.PeriNormArgs()
            a.rows, a.d, a.eps, a.scale, a.rows_per_gate = rows, d, 1e-5, 0.5, per
            a.ld_x = a.ld_f = a.ld_d_out = a.ld_dn = d
            for i, name in enumerate(("x", "f", "w_post", "w_pre", "d_out", "dn", "x_out", "n_out", "df", "d_w_post", "d_w_pre", "gate", "d_gate")):
                if name not in drop and (per or "gate" not in name):
                    setattr(a, name, B + (i << 42))
            for k, v in kw.items():
                setattr(a, k, v)
            return a
        def backward(a):
            c.mtdao_peri_norm_backward(a, B << 8, c.mtdao_peri_norm_backward_workspace_bytes(a), None)
"""


@pytest.mark.parametrize("more", ["", ", drop=('w_pre', 'dn')", ", drop=('f', 'w_post', 'df', 'd_w_post')", ", 5"])
def test_boundary_gradients_of_no_rows(run, more):
    """Only the sums over rows are written."""
    launches, _ = run(PERI + f"        backward(peri(0, 64{more}))\n")
    assert launches == [("k_peri_columns", (2, 2, 1), 1024, 0)]


@pytest.mark.parametrize("rows", [1, 7, 5000])
@pytest.mark.parametrize("per", [2 ** 63 - 1, 2 ** 62, 2 ** 31])
def test_gates_of_more_rows_than_there_are(run, rows, per):
    """... are one gate: their gradient is summed as that of exactly the rows."""
    launches, _ = run(PERI + f"""
        backward(peri({rows}, 64, {per}))
        backward(peri({rows}, 64, {rows}))
        c.mtdao_peri_norm(peri({rows}, 64, {per}), None)
    """)
    assert names(launches) == ["k_peri_norm_backward", "k_peri_columns"] * 2 + ["k_peri_norm"]
    assert launches[:2] == launches[2:4] and launches[1][1] == (2, 3, 1)


# ------------------------------------------------------------------- AdamW

ADAMW = """
        B, AT = 1 << 40, 1 << 30
        def adamw(numels, bits=32, **kw):
            cfg = c.AdamwConfig(0, 0, bits, len(numels), 0.9, 0.95, 1e-8, 0.0, 0)
            rows = (c.AdamwTensor * len(numels))()
            for i, n in enumerate(numels):
                at = B + i * AT
                rows[i] = c.AdamwTensor(at, at + (1 << 26), at + (2 << 26), at + (3 << 26), at + (4 << 26), at + (5 << 26), n, 0.1)
            for k, v in kw.items():
                name, _, i = k.partition("__")
                setattr(rows[int(i)] if i else cfg, name, v)
            return c.mtdao_adamw_init(cfg, rows, B << 1, c.mtdao_adamw_workspace_bytes(cfg, rows), None)
"""


def test_adamw_gradients_and_what_is_written(run):
    """On its own tensor, element on element, a gradient is taken (as before); on
    others, or shifted, it is refused, at construction and later."""
    launches, said = run(ADAMW + """
        for kw in (dict(g__0=B), dict(g__1=B + AT + (2 << 26)), dict(g__1=B + AT + (3 << 26)), dict(g__0=B + 4000), dict(g__1=B + AT - 4000)):
            c.mtdao_adamw_destroy(adamw([1000, 1000, 0], **kw))
        h = adamw([1000, 1000, 0])
        good = [B + (1 << 26), B + AT + (1 << 26), None]
        for i, g in ((0, B), (1, B + AT), (0, B + AT), (1, B + 4), (0, B + AT - 3996), (1, B + (2 << 26)), (2, B)):
            grads = list(good)
            grads[i] = g
            try:
                c.mtdao_adamw_set_grads(h, grads, None)
                say("taken")
            except abi.MtdaoError as e:
                say(str(e))
    """)
    assert names(launches) == ["k_adamw_table"] * 6 + ["k_adamw_grads"] * 3
    assert [s if s == "taken" else "overlaps" in s for s in said] == ["taken"] * 2 + [True] * 4 + ["taken"]


# -------------------------------------------------------------- largest launches


@pytest.mark.parametrize("rows,d", [(1, 64), ((1 << 21) + 1, 2048), ((1 << 23) + 1, 64), ((1 << 26) + 5, 8), (1 << 24, 8192), (1 << 30, 512), ((1 << 38) + 1, 1)])
def test_boundaries_of_many_rows_fit_a_launch(run, rows, d):
    """Fewer than 2^32 threads along x, every row in a workgroup, no row of
    workgroups without one."""
    launches, _ = run(PERI + f"        c.mtdao_peri_norm(peri({rows}, {d}, ld_f={d}), None)\n")
    (name, (x, y, z), threads, _), = launches
    per = 4 if d <= 512 else 1
    assert name == "k_peri_norm" and z == 1 and x * threads < 1 << 32 and y <= 65535
    assert x * y * per >= rows > x * (y - 1) * per


@pytest.mark.parametrize("rows,cols", [(5, 300), ((1 << 26) + 1, 8), (1 << 22, 8192), (3, 1 << 22), ((1 << 31) - 1, 100)])
def test_quantized_rows_fit_a_launch(run, rows, cols):
    launches, _ = run(f"""
        B = 1 << 40
        c.mtdao_quantize8(B, 1, {cols}, c.Matrix8(B << 8, B << 10, {rows}, {cols}, -(-{cols} // 128) * 128, 4 * {rows}, 1), None, None)
    """)
    (name, (x, y, z), threads, _), = launches
    groups, fours = -(-cols // 512), -(-rows // 4)
    assert name == "k_quantize8_rows" and z == 1 and x % groups == 0 and x * threads < 1 << 32 and y <= 65535
    assert x // groups * y >= fours > x // groups * (y - 1)


@pytest.mark.parametrize("n", [100, (1 << 25) + 3, (1 << 27) + 1, (1 << 31) - 1])
def test_products_of_many_columns_and_few_rows_fit_a_launch(run, n):
    launches, _ = run(f"""
        B = 1 << 40
        matrix = lambda rows, at: c.Matrix8(at, at + (1 << 39), rows, 128, 128, 4 * rows, 1)
        for m in (8, 64):
            c.mtdao_product8(matrix(m, B), matrix({n}, B << 2), B << 4, 1, {n}, False, None, 0, None)
    """)
    assert len(launches) == 2
    for (name, (x, y, z), threads, _), cols in zip(launches, (16, 32 if n > 4096 else 16)):
        assert name == "k_product8_few" and z == 1 and x * threads < 1 << 32 and y <= 65535
        assert x * y * cols >= n > x * (y - 1) * cols
