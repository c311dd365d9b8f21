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
