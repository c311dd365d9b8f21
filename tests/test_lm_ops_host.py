"""Host-side checks of the orthogonalised updates, the embedding and the cross
entropy (no GPU): structures, workspaces, and what the entry points refuse before
anything is enqueued (device addresses that are never dereferenced)."""

import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

from paper_2510_05361_amd import build, mtdao as abi, mtdao_ops as c, ops

HEADER = os.path.join(build.ROOT, "include", "mtdao_ops.h")
BASE = 1 << 40
NAN, INF = float("nan"), float("inf")


def test_constants_match_the_header():
    text = open(HEADER).read()
    for name in ("MTDAO_MUON_MAX_SIDE", "MTDAO_MUON_MAX_STEPS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(c, name)
    for name in ("MTDAO_LOSS_NONE", "MTDAO_LOSS_SUM", "MTDAO_LOSS_MEAN"):
        assert int(re.search(rf"\b{name}\s*=\s*(\d+)", text).group(1)) == getattr(c, name)


def test_structures_have_the_headers_layout(tmp_path):
    pairs = [("mtdao_muon_matrix", c.MuonMatrix), ("mtdao_muon_config", c.MuonConfig), ("mtdao_cross_entropy_args", c.CrossEntropyArgs)]
    lines = [f'printf("%zu", sizeof({n}));' + "".join(f'printf(" %zu", offsetof({n}, {f}));' for f, _ in s._fields_) + 'printf("\\n");'
             for n, s in pairs]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "mtdao_ops.h"\nint main(void) {' + "".join(lines) + "return 0;}")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), "-o", str(exe), str(src)], check=True)
    got = [list(map(int, l.split())) for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    assert got == [[ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_] for _, s in pairs]
    assert c.PACKED_LOSS.size == ctypes.sizeof(c.CrossEntropyArgs)


def refused(code, call, *args):
    with pytest.raises(abi.MtdaoError) as e:
        call(*args)
    assert e.value.code == code and str(e.value), e.value


# -------------------------------------------------------------------- updates


@pytest.mark.parametrize("batch,rows,cols,code", [(-1, 4, 4, -1), ((1 << 20) + 1, 4, 4, -1), (1, -1, 4, -1), (1, 4, -1, -1), (1, 16385, 16385, -1),
                                                  (1, 3, (1 << 20) + 1, -1), (1, 1 << 62, 1 << 62, -1)])
def test_orthogonalize_refuses_sizes(batch, rows, cols, code):
    refused(code, c.mtdao_orthogonalize_workspace_bytes, batch, rows, cols)
    refused(code, c.mtdao_orthogonalize, BASE, 0, batch, rows, cols, BASE << 1, 0, 5, 1e-7, BASE << 2, 1 << 40, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(dtype=2), -1), (dict(out_dtype=-1), -1), (dict(steps=0), -1), (dict(steps=65), -1),
    (dict(eps=-1e-9), -1), (dict(eps=NAN), -1), (dict(eps=INF), -1), (dict(x=BASE + 2), -2), (dict(out=(BASE << 1) + 1), -2), (dict(ws=None), -5),
    (dict(need=100), -5), (dict(ws=(BASE << 2) + 128), -2), (dict(out=BASE + 400), -1), (dict(out=BASE, out_dtype=1), -1)])
def test_orthogonalize_refuses(kw, code):
    a = dict(x=BASE, dtype=0, out=BASE << 1, out_dtype=0, steps=5, eps=1e-7, ws=BASE << 2, need=c.mtdao_orthogonalize_workspace_bytes(2, 130, 140))
    a.update(kw)
    refused(code, c.mtdao_orthogonalize, a["x"], a["dtype"], 2, 130, 140, a["out"], a["out_dtype"], a["steps"], a["eps"], a["ws"], a["need"], None)


def test_nothing_to_orthogonalize():
    for batch, rows, cols in ((0, 5, 5), (3, 0, 5), (3, 5, 0)):
        assert c.mtdao_orthogonalize_workspace_bytes(batch, rows, cols) == 0
        c.mtdao_orthogonalize(None, 0, batch, rows, cols, None, 0, 5, 1e-7, None, 0, None)
    assert c.mtdao_orthogonalize_workspace_bytes(1000, 64, 256) == c.mtdao_orthogonalize_workspace_bytes(1, 256, 64) == 0  # one workgroup each
    assert c.mtdao_orthogonalize_workspace_bytes(1, 65, 65) > 0 and c.mtdao_orthogonalize_workspace_bytes(1, 1, 257) > 0


def muon_case(n=3, **kw):
    cfg = c.MuonConfig(abi.MTDAO_F32, abi.MTDAO_F32, n, 1, 5, 0, 0.95, 1e-7)
    rows = (c.MuonMatrix * max(n, 1))()
    for i in range(n):
        at = BASE + i * (1 << 30)
        rows[i] = c.MuonMatrix(at, at + (1 << 26), at + (2 << 26), 20, 50, 0.1, 1.0)
    for k, v in kw.items():
        name, _, i = k.partition("__")
        setattr(rows[int(i)] if i else cfg, name, v)
    return cfg, rows


MUON_BAD = [
    (dict(param_dtype=2), -1), (dict(grad_dtype=-1), -1), (dict(n_matrices=0), -1), (dict(n_matrices=(1 << 20) + 1), -1), (dict(steps=0), -1),
    (dict(steps=65), -1), (dict(momentum=1.0), -1), (dict(momentum=-0.1), -1), (dict(momentum=NAN), -1), (dict(eps=-1.0), -1), (dict(eps=INF), -1),
    (dict(rows__1=-1), -1), (dict(cols__1=-1), -1), (dict(rows__1=1 << 40), -1), (dict(weight_decay__0=-0.1), -1), (dict(weight_decay__0=NAN), -1),
    (dict(factor__2=NAN), -1), (dict(factor__2=INF), -1), (dict(p__2=None), -1), (dict(g__0=None), -1), (dict(m__0=None), -1), (dict(p__0=BASE + 2), -2),
    (dict(g__1=BASE + 1), -2), (dict(m__0=BASE + (1 << 27) + 2), -2), (dict(p__1=BASE), -1), (dict(m__0=BASE + 3996), -1), (dict(g__0=BASE), -1),
    (dict(g__0=BASE + (2 << 26)), -1), (dict(g__1=BASE + 3996), -1), (dict(grad_dtype=1, g__1=BASE + 3998), -1),
]


@pytest.mark.parametrize("kw,code", MUON_BAD, ids=[str(k) for k, _ in MUON_BAD])
def test_muon_refuses(kw, code):
    cfg, rows = muon_case(**kw)
    refused(code, c.mtdao_muon_init, cfg, rows, BASE << 1, 1 << 40, None)


def test_muon_refuses_workspaces():
    cfg, rows = muon_case()
    need = c.mtdao_muon_workspace_bytes(cfg, rows)
    refused(-5, c.mtdao_muon_init, cfg, rows, None, need, None)
    refused(-5, c.mtdao_muon_init, cfg, rows, BASE << 1, need - 1, None)
    refused(-2, c.mtdao_muon_init, cfg, rows, (BASE << 1) + 64, need, None)
    assert c.lib().mtdao_muon_step(None, 0.1, None) == -1 and c.lib().mtdao_muon_set_grads(None, None, None) == -1
    c.lib().mtdao_muon_destroy(None)


def test_muon_workspaces_stay_small():
    """Matrices go through in groups: a thousand large ones take no more than a few."""
    sizes = []
    for n in (4, 400):
        cfg, rows = muon_case(n)
        for r in rows:
            r.rows, r.cols = 2048, 8192
        sizes.append(c.mtdao_muon_workspace_bytes(cfg, rows))
    assert sizes[0] < sizes[1] < 6 << 30


# ------------------------------------------------------------------ embedding


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), -1), (dict(n=(1 << 30) + 1), -1), (dict(rows=-1), -1), (dict(rows=(1 << 30) + 1), -1), (dict(d=0), -1), (dict(d=(1 << 20) + 1), -1),
    (dict(bits=16), -1), (dict(tokens=None), -1), (dict(tokens=BASE + 4), -2), (dict(w=None), -1), (dict(w=(BASE << 1) + 1), -2), (dict(w_type=3), -1),
    (dict(ld=15), -1), (dict(ld=1 << 40), -1), (dict(scale=NAN), -1), (dict(scale=INF), -1), (dict(y=None), -1), (dict(y=(BASE << 2) + 2), -2),
    (dict(y_type=-1), -1), (dict(ld_y=3), -1)])
def test_embedding_refuses(kw, code):
    a = dict(tokens=BASE, bits=64, n=10, w=BASE << 1, w_type=1, rows=100, d=16, ld=16, scale=1.0, y=BASE << 2, y_type=0, ld_y=16)
    a.update(kw)
    refused(code, c.mtdao_embedding, *(a[k] for k in ("tokens", "bits", "n", "w", "w_type", "rows", "d", "ld", "scale", "y", "y_type", "ld_y")), None)
    if set(kw) & {"n", "rows", "d", "bits", "tokens", "scale"} or kw == dict(y_type=-1):
        need = 1 << 40
        refused(code, c.mtdao_embedding_backward, a["y"], a["y_type"], a["ld_y"], a["tokens"], a["bits"], a["n"], a["scale"], BASE << 3, a["rows"], a["d"],
                a["d"], False, BASE << 4, need, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), -1), (dict(dy=BASE + 1), -2), (dict(ld_dy=7), -1), (dict(dw=None), -1), (dict(dw=(BASE << 1) + 2), -2), (dict(ld_dw=9), -1),
    (dict(dw=BASE + 64), -1), (dict(dw=(BASE << 2) + 16), -1), (dict(ws=None), -5), (dict(need=-1), -5), (dict(ws=(BASE << 3) + 16), -2)])
def test_embedding_backward_refuses(kw, code):
    need = c.mtdao_embedding_backward_workspace_bytes(10, 100, 16)
    a = dict(dy=BASE, ld_dy=16, tokens=BASE << 2, dw=BASE << 1, ld_dw=16, ws=BASE << 3, need=0)
    a.update(kw)
    refused(code, c.mtdao_embedding_backward, a["dy"], 1, a["ld_dy"], a["tokens"], 64, 10, 1.0, a["dw"], 100, 16, a["ld_dw"], False, a["ws"],
            need + a["need"], None)


# -------------------------------------------------------------- cross entropy


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(rows=(1 << 31) + 1), -1), (dict(cols=0), -1), (dict(cols=(1 << 31) + 1), -1), (dict(dtype=2), -1), (dict(target_bits=8), -1),
    (dict(reduction=3), -1), (dict(z_loss=NAN), -1), (dict(scale=INF), -1), (dict(ld_logits=49), -1), (dict(ld_d=49), -1), (dict(ld_logits=1 << 40), -1),
    (dict(logits=None), -1), (dict(targets=None), -1), (dict(logits=BASE + 2), -2), (dict(targets=(BASE << 1) + 4), -2), (dict(d_loss=2), -2),
    (dict(losses=2), -2), (dict(loss=2), -2), (dict(d_logits=(BASE << 2) + 2), -2), (dict(d_logits=BASE + 400), -1), (dict(d_logits=BASE, ld_d=60), -1),
    (dict(d_logits=BASE << 1), -1), (dict(reduction=0), -1), (dict(loss=None, losses=None, d_logits=None), -1)])
def test_cross_entropy_refuses(kw, code):
    a = c.CrossEntropyArgs(7, 50, 50, 50, 0, 64, 2, 0.0, 1.0, 0, BASE, BASE << 1, None, None, BASE << 3, BASE << 2)
    for k, v in kw.items():
        setattr(a, k, v)
    refused(code, c.mtdao_cross_entropy, a, BASE << 4, 1 << 40, None)


@pytest.mark.parametrize("kw", [
    dict(losses=BASE + 4), dict(losses=(BASE << 1) + 8), dict(losses=(BASE << 2) + 1396), dict(losses=BASE << 5), dict(losses=(BASE << 5) - 24),
    dict(loss=BASE), dict(loss=(BASE << 1) + 52), dict(loss=(BASE << 2) + 8), dict(loss=BASE << 5), dict(losses=BASE << 3, loss=(BASE << 3) + 24),
    dict(d_loss=(BASE << 2) + 1396), dict(reduction=0, loss=None, losses=(BASE << 5) + 24), dict(reduction=0, loss=None, d_loss=(BASE << 2) - 24)])
def test_cross_entropy_refuses_losses_that_overlap(kw):
    a = c.CrossEntropyArgs(7, 50, 50, 50, 0, 64, 2, 0.0, 1.0, 0, BASE, BASE << 1, BASE << 5, None, BASE << 3, BASE << 2)
    for k, v in kw.items():
        setattr(a, k, v)
    refused(-1, c.mtdao_cross_entropy, a, BASE << 4, 1 << 40, None)


def test_cross_entropy_refuses_workspaces():
    a = c.CrossEntropyArgs(7, 50, 50, 50, 0, 64, 2, 0.0, 1.0, 0, BASE, BASE << 1, None, None, BASE << 3, BASE << 2)
    need = c.mtdao_cross_entropy_workspace_bytes(a)
    refused(-5, c.mtdao_cross_entropy, a, None, need, None)
    refused(-5, c.mtdao_cross_entropy, a, BASE << 4, need - 1, None)
    refused(-2, c.mtdao_cross_entropy, a, (BASE << 4) + 8, need, None)


# ---------------------------------------------------------------------- torch


def test_tensors_on_the_cpu_are_refused():
    x, ids = torch.randn(4, 6), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.orthogonalize(x), lambda: ops.Muon([x], [x]), lambda: ops.embedding(ids, x), lambda: ops.embedding_backward(x, ids, 9),
                 lambda: ops.cross_entropy(x, ids), lambda: ops.cross_entropy_step(x, ids), lambda: ops.cross_entropy_backward(None, x, ids)):
        with pytest.raises(ValueError, match="the GPU only"):
            call()


def test_arguments_that_do_not_fit():
    x, ids = torch.randn(4, 6), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="matrices"):
        ops.orthogonalize(torch.randn(5))
    with pytest.raises(ValueError, match="no parameters"):
        ops.Muon([], [])
    with pytest.raises(ValueError, match="requires a gradient"):
        ops.orthogonalize(x.clone().requires_grad_())
    with pytest.raises(ValueError, match="tokens"):
        ops.embedding_backward(x, ids[:3], 9)
    with pytest.raises(ValueError, match="needs dw"):
        ops.embedding_backward(x, ids, 9, accumulate=True)
    for dw in (torch.zeros(9, 5), torch.zeros(9, 6, dtype=torch.bfloat16), torch.zeros(6, 9).t()):
        with pytest.raises(ValueError, match="dw"):
            ops.embedding_backward(x, ids, 9, dw=dw)
    with pytest.raises(ValueError, match="reduction"):
        ops.cross_entropy(x, ids, reduction="max")
    with pytest.raises(ValueError, match="targets"):
        ops.cross_entropy(x, ids[:3])
    with pytest.raises(ValueError, match="targets"):
        ops.cross_entropy(torch.empty(4, 0), ids)
    for d in (torch.zeros(4), torch.zeros((), dtype=torch.float64)):
        with pytest.raises(ValueError, match="d_loss"):
            ops.cross_entropy_backward(d, x, ids)
    assert math.isfinite(float(x.sum()))
