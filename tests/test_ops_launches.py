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


ANY_SIZES = r"""
        import random
        rng = random.Random(5)
        B, MOST = 1 << 40, (1 << 63) - 1
        up = lambda n, m: -(-n // m) * m if n < 1 << 60 else 0

        def size():
            return rng.choice([0, 1, 2, 3, 7, 64, 127, 128, 129, 4096, 8192, 8193, 1 << 22, (1 << 22) + 1, (1 << 31) - 1, 1 << 31, 1 << 40, 1 << 62, MOST, -1,
                               rng.randrange(1, 1 << 20)])

        def matrix(rows, cols, at, scale_rows=1, ld=None):
            return c.Matrix8(at, at + (1 << 52), rows, cols, max(128, up(cols, 128)) if ld is None else ld, 4 * up(rows, scale_rows) // scale_rows, scale_rows)

        def boundary():
            a = c.PeriNormArgs()
            a.rows, a.d, a.rows_per_gate = size(), rng.choice([size(), 64, 768, 2048]), size()
            a.kind, a.stream_dtype, a.branch_dtype, a.weight_dtype = (rng.choice([0, 1]) for _ in range(4))
            a.eps, a.scale = 1e-5, 1.0
            a.ld_x, a.ld_f, a.ld_d_out, a.ld_dn = (rng.choice([a.d, a.d, size()]) for _ in range(4))
            for i, name in enumerate(("x", "f", "w_post", "w_pre", "gate", "d_out", "dn", "x_out", "n_out", "df", "d_w_post", "d_w_pre", "d_gate")):
                if rng.random() < 0.85:
                    setattr(a, name, B + (i << 44) + rng.choice([0, 0, 0, 0, 2, 4]))
            if rng.random() < 0.5:
                c.mtdao_peri_norm(a, None)
            else:
                c.mtdao_peri_norm_backward(a, B << 10, c.mtdao_peri_norm_backward_workspace_bytes(a), None)

        def quantize():
            r, k, s = size(), size(), rng.choice([1, 128])
            q, qt = matrix(r, k, B, s, rng.choice([up(k, 128), size()])), matrix(k, r, B << 8, s)
            c.mtdao_quantize8(B << 14, rng.choice([0, 1]), rng.choice([k, size()]), rng.choice([q, None]), rng.choice([qt, None]), None)

        def product():
            m, n, k = size(), size(), size()
            need = c.mtdao_product8_workspace_bytes(m, n, k)
            c.mtdao_product8(matrix(m, k, B), matrix(n, k, B << 13), B << 17, rng.choice([0, 1]), rng.choice([n, size()]), 0, B << 18, need, None)

        def linear():
            m, n, k = (rng.choice([0, 1, 5, 16, 17, 64, 65, 300, 4000, 1 << 22]) for _ in range(3))
            f, b = c.mtdao_linear8_workspace_bytes(m, n, k)
            t = rng.choice([0, 1])
            c.mtdao_linear8(B << 14, t, m, k, matrix(n, k, B, 128), B << 15, rng.choice([0, 1]), n, B << 16, f, None)
            c.mtdao_linear8_backward(B << 14, B << 15, t, m, n, k, matrix(k, n, B, 128), B << 16, k, B << 17, k, rng.choice([0, 1]), B << 18, b, None)

        def adamw():
            n = rng.randrange(1, 5)
            cfg = c.AdamwConfig(rng.choice([0, 1]), rng.choice([0, 1]), rng.choice([32, 8]), n, 0.9, 0.95, rng.choice([0, 1e-8, 1e-40]), rng.choice([0, 1.0]),
                                rng.choice([0, 5, MOST - 10]))
            rows = (c.AdamwTensor * n)(*(c.AdamwTensor(*(B + (i << 46) + (j << 43) for j in range(6)), size(), 0.1) for i in range(n)))
            need = c.mtdao_adamw_workspace_bytes(cfg, rows)
            h = c.mtdao_adamw_init(cfg, rows, B << 20, need, None)
            c.mtdao_adamw_step(h, 1e-3, None)
            c.mtdao_adamw_destroy(h)

        taken = refused = 0
        for _ in range(6000):
            try:
                rng.choice([boundary, boundary, quantize, product, linear, adamw])()
                taken += 1
            except abi.MtdaoError:
                refused += 1
        say([taken, refused])
"""


def test_any_sizes_are_refused_or_fit_their_launches(run):
    launches, said = run(ANY_SIZES)
    assert min(said[0]) > 1000, said
    for name, (x, y, z), threads, _ in launches:
        assert x >= 1 and y >= 1 and z == 1 and x * threads < 1 << 32 and y <= 65535, (name, x, y, threads)
