"""Host-side checks of include/mtdao_ops.h (no GPU): exported symbols, the
binding's structures and constants, and what the entry points refuse before
anything is enqueued (device addresses that are never dereferenced)."""

import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2510_05361_amd import build, mtdao as abi, mtdao_ops as c, ops

HEADER = os.path.join(build.ROOT, "include", "mtdao_ops.h")
BASE = 1 << 40


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(mtdao_\w+)\s*\(", text)))
    assert len(names) >= 12, names
    for n in names:
        assert hasattr(c.lib(), n), n


def test_constants_match_the_header():
    text = open(HEADER).read()
    for name in ("MTDAO_BLOCK8", "MTDAO_PERI_MAX_D"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(c, name)
    for name in ("MTDAO_NORM_RMS", "MTDAO_NORM_LAYER"):
        assert int(re.search(rf"\b{name}\s*=\s*(\d+)", text).group(1)) == getattr(c, name)


def test_structures_have_the_headers_layout(tmp_path):
    """Sizes and last offsets as a C compiler sees them (the header is C)."""
    pairs = [("mtdao_adamw_tensor", c.AdamwTensor), ("mtdao_adamw_config", c.AdamwConfig),
             ("mtdao_peri_norm_args", c.PeriNormArgs), ("mtdao_matrix8", c.Matrix8)]
    lines = [f'printf("%zu %zu\\n", sizeof({n}), offsetof({n}, {s._fields_[-1][0]}));' for n, s in pairs]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "mtdao_ops.h"\nint main(void) {' + "".join(lines) + "return 0;}")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), "-o", str(exe), str(src)], check=True)
    got = [tuple(map(int, l.split())) for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    assert got == [(ctypes.sizeof(s), getattr(s, s._fields_[-1][0]).offset) for _, s in pairs]


# ------------------------------------------------------------------- AdamW


def adamw_case(n=3, bits=32, **kw):
    cfg = c.AdamwConfig(abi.MTDAO_F32, abi.MTDAO_F32, bits, n, 0.9, 0.95, 1e-8, 0.0, 0)
    rows = (c.AdamwTensor * max(n, 1))()
    for i in range(n):
        at = BASE + i * (1 << 30)
        rows[i] = c.AdamwTensor(at, at + (1 << 26), at + (2 << 26), at + (3 << 26), at + (4 << 26), at + (5 << 26), 1000, 0.1)
    for k, v in kw.items():
        name, _, i = k.partition("__")
        setattr(rows[int(i)] if i else cfg, name, v)
    return cfg, rows


ADAMW_BAD = [
    (dict(param_dtype=2), -1), (dict(grad_dtype=-1), -1), (dict(state_bits=16), -1), (dict(n_tensors=0), -1),
    (dict(beta1=1.0), -1), (dict(beta1=float("nan")), -1), (dict(beta2=-0.1), -1), (dict(eps=-1e-8), -1),
    (dict(eps=float("inf")), -1), (dict(max_norm=float("nan")), -1), (dict(start_step=-1), -1),
    (dict(numel__1=-1), -1), (dict(numel__1=1 << 41), -1), (dict(weight_decay__0=-0.1), -1),
    (dict(weight_decay__0=float("nan")), -1), (dict(p__2=None), -1), (dict(g__0=None), -1), (dict(m__0=None), -1),
    (dict(v__1=None), -1), (dict(p__0=BASE + 2), -2), (dict(g__1=BASE + 1), -2), (dict(m__0=BASE + 8), -2),
    (dict(v__0=BASE + 4), -2), (dict(p__1=BASE), -1), (dict(m__0=BASE + 2008), -2), (dict(m__0=BASE + 1600), -1),
    (dict(bits=8, m_scale__0=None), -1), (dict(bits=8, v_scale__2=None), -1),
]


@pytest.mark.parametrize("kw,code", ADAMW_BAD, ids=[str(k) for k, _ in ADAMW_BAD])
def test_adamw_refuses(kw, code):
    cfg, rows = adamw_case(**kw)
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_adamw_init(cfg, rows, BASE << 1, 1 << 30, None)
    assert e.value.code == code
    assert abi.mtdao_last_error(None) != ""


def test_adamw_workspace():
    cfg, rows = adamw_case(max_norm=1.0)
    need = c.mtdao_adamw_workspace_bytes(cfg, rows)
    assert need >= 3 * 72 + 3 * 4 + 3 * 8
    for ws, size, code in ((None, 1 << 20, -5), (BASE << 1, need - 1, -5), ((BASE << 1) + 128, need, -2)):
        with pytest.raises(abi.MtdaoError) as e:
            c.mtdao_adamw_init(cfg, rows, ws, size, None)
        assert e.value.code == code
    assert c.mtdao_adamw_step_count(None) == -1
    c.mtdao_adamw_destroy(None)
    for call in (lambda: c.mtdao_adamw_step(None, 1e-3, None), lambda: c.mtdao_adamw_set_grads(None, [1], None)):
        with pytest.raises(abi.MtdaoError) as e:
            call()
        assert e.value.code == abi.MTDAO_ERR_INVALID_ARG


# -------------------------------------------------------------- Peri-LN


def peri_case(backward=False, **kw):
    a = c.PeriNormArgs()
    a.rows, a.d, a.eps, a.scale, a.rows_per_gate = 10, 64, 1e-5, 0.5, 4
    a.ld_x = a.ld_f = a.ld_d_out = a.ld_dn = 64
    names = ["x", "f", "w_post", "w_pre", "gate", "x_out"] + (["d_out", "dn", "df", "d_w_post", "d_w_pre", "d_gate"] if backward else ["n_out"])
    for i, n in enumerate(names):
        setattr(a, n, BASE + i * (1 << 20))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


PERI_BAD = [(dict(rows=-1), -1), (dict(d=0), -1), (dict(d=c.MTDAO_PERI_MAX_D + 1), -1), (dict(kind=2), -1),
            (dict(stream_dtype=2), -1), (dict(branch_dtype=3), -1), (dict(weight_dtype=-1), -1),
            (dict(stream_dtype=1, branch_dtype=0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
            (dict(scale=float("inf")), -1), (dict(rows_per_gate=0), -1), (dict(f=None), -1), (dict(f=None, gate=None, w_pre=None), -1),
            (dict(w_post=None), -1), (dict(x=None), -1), (dict(x_out=None), -1), (dict(ld_x=63), -1), (dict(ld_f=8), -1),
            (dict(ld_x=1 << 41), -1), (dict(rows=1 << 41), -1), (dict(x=BASE + 1), -2), (dict(w_pre=BASE + 2), -2),
            (dict(x_out=BASE + 4), -1)]


@pytest.mark.parametrize("kw,code", PERI_BAD + [(dict(n_out=None), -1), (dict(n_out=BASE + 5 * (1 << 20)), -1)], ids=str)
def test_peri_norm_refuses(kw, code):
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_peri_norm(peri_case(**kw), None)
    assert e.value.code == code


@pytest.mark.parametrize("kw,code", PERI_BAD + [(dict(df=None), -1), (dict(d_w_post=None), -1), (dict(d_w_pre=None), -1),
                                                (dict(d_gate=None), -1), (dict(d_gate=BASE + 2), -2), (dict(ld_dn=1), -1),
                                                (dict(df=BASE + 5 * (1 << 20)), -1), (dict(dn=BASE + 3), -2)], ids=str)
def test_peri_norm_backward_refuses(kw, code):
    a = peri_case(True, **kw)
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_peri_norm_backward(a, BASE << 1, 1 << 30, None)
    assert e.value.code == code


def test_peri_norm_workspace():
    a = peri_case(True)
    need = c.mtdao_peri_norm_backward_workspace_bytes(a)
    assert need >= 3 * 64 * 4
    for ws, size, code in ((None, 0, -5), (BASE << 1, need - 1, -5), ((BASE << 1) + 4, need, -2)):
        with pytest.raises(abi.MtdaoError) as e:
            c.mtdao_peri_norm_backward(a, ws, size, None)
        assert e.value.code == code
    c.mtdao_peri_norm(peri_case(rows=0, x=None, f=BASE, n_out=None), None)  # no rows: nothing to do


# ------------------------------------------------------------ 8-bit product


def matrix(rows, cols, at=BASE, scale_rows=1, **kw):
    ld = -(-cols // 128) * 128
    m = c.Matrix8(at, at + (1 << 32), rows, cols, ld, 4 * -(-rows // scale_rows), scale_rows)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


QUANT_BAD = [
    (dict(), None, None, -1), (dict(dtype=2), matrix(4, 200), None, -1), (dict(ld=199), matrix(4, 200), None, -1),
    (dict(x=None), matrix(4, 200), None, -1), (dict(x=(BASE << 1) + 2), matrix(4, 200), None, -2),
    (dict(), matrix(4, 200, ld=200), None, -1), (dict(), matrix(4, 200, scale_ld=2), None, -1),
    (dict(), matrix(4, 200, scale_rows=64), None, -1), (dict(), matrix(4, 200, codes=None), None, -1),
    (dict(), matrix(4, 200, codes=BASE + 8), None, -2), (dict(), matrix(4, 200, scales=BASE + 2), None, -2),
    (dict(), matrix(-1, 200), None, -1), (dict(), matrix(4, (1 << 22) + 1), None, -1),
    (dict(), matrix(4, 200), matrix(200, 5), -1), (dict(), matrix(4, 200), matrix(200, 4, scale_rows=128), -1),
    (dict(x=BASE + 512), matrix(4, 200), None, -1),
]


@pytest.mark.parametrize("kw,q,qt,code", QUANT_BAD, ids=[str(i) for i in range(len(QUANT_BAD))])
def test_quantize8_refuses(kw, q, qt, code):
    a = {"x": BASE << 1, "dtype": 0, "ld": 200, **kw}
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_quantize8(a["x"], a["dtype"], a["ld"], q, qt, None)
    assert e.value.code == code


B2 = BASE + (1 << 34)
PRODUCT_BAD = [
    (dict(), matrix(4, 200), matrix(5, 201, B2), -1), (dict(c_dtype=2), matrix(4, 200), matrix(5, 200, B2), -1),
    (dict(accumulate=True, c_dtype=1), matrix(4, 200), matrix(5, 200, B2), -1), (dict(ldc=4), matrix(4, 200), matrix(5, 200, B2), -1),
    (dict(c=None), matrix(4, 200), matrix(5, 200, B2), -1), (dict(c=(BASE << 1) + 2), matrix(4, 200), matrix(5, 200, B2), -2),
    (dict(c=B2), matrix(4, 200), matrix(5, 200, B2), -1), (dict(), matrix(4, 200, codes=None), matrix(5, 200, B2), -1),
    (dict(), matrix(4, 200), matrix(5, 200, B2, scale_ld=8), -1),
]


@pytest.mark.parametrize("kw,a,b,code", PRODUCT_BAD, ids=[str(i) for i in range(len(PRODUCT_BAD))])
def test_product8_refuses(kw, a, b, code):
    k = {"c": BASE << 1, "c_dtype": 0, "ldc": 5, "accumulate": False, **kw}
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_product8(a, b, k["c"], k["c_dtype"], k["ldc"], k["accumulate"], BASE << 2, 1 << 40, None)
    assert e.value.code == code


def test_product8_without_rows_does_nothing():
    c.mtdao_product8(matrix(0, 200), matrix(5, 200, B2), None, 0, 5, False, None, 0, None)
    c.mtdao_quantize8(None, 0, 0, matrix(3, 0), None, None)
    with pytest.raises(abi.MtdaoError):
        c.mtdao_product8_workspace_bytes(-1, 1, 1)


LINEAR_BAD = [
    (dict(dtype=2), -1), (dict(x=None), -1), (dict(x=(BASE << 1) + 2), -2), (dict(ld=199), -1), (dict(rows=-1), -1),
    (dict(rows=(1 << 22) + 1), -1), (dict(y=None), -1), (dict(y_dtype=3), -1), (dict(ldy=4), -1), (dict(y=BASE << 1), -1),
    (dict(y=BASE), -1), (dict(w=matrix(5, 200, codes=None)), -1), (dict(w=matrix(5, 200, scale_ld=8)), -1), (dict(workspace=None), -5),
    (dict(size=-1), -5), (dict(workspace=(BASE << 3) + 4), -2),
]


@pytest.mark.parametrize("kw,code", LINEAR_BAD, ids=[str(i) for i in range(len(LINEAR_BAD))])
def test_linear8_refuses(kw, code):
    a = {"x": BASE << 1, "dtype": 0, "rows": 40, "ld": 200, "w": matrix(5, 200), "y": BASE << 2, "y_dtype": 0, "ldy": 5,
         "workspace": BASE << 3, "size": 0, **kw}
    need = c.mtdao_linear8_workspace_bytes(40, 5, 200)[0] + a.pop("size")
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_linear8(*a.values(), need, None)
    assert e.value.code == code


LINEAR_BACKWARD_BAD = [
    (dict(dtype=2), -1), (dict(dy=None), -1), (dict(x=None), -1), (dict(dy=(BASE << 1) + 2), -2), (dict(ld_dy=4), -1), (dict(ld_x=199), -1),
    (dict(rows=-1), -1), (dict(rows=(1 << 22) + 1), -1), (dict(dx=None), -1), (dict(dw=None), -1), (dict(ld_dx=199), -1), (dict(ld_dw=199), -1),
    (dict(dw=(BASE << 4) + 2), -2), (dict(dx=BASE << 4), -1), (dict(dx=BASE << 1), -1), (dict(dw=BASE << 2), -1), (dict(dw=BASE), -1),
    (dict(wt=matrix(200, 5, codes=None)), -1), (dict(workspace=None), -5), (dict(size=-1), -5), (dict(workspace=(BASE << 5) + 4), -2),
]


@pytest.mark.parametrize("kw,code", LINEAR_BACKWARD_BAD, ids=[str(i) for i in range(len(LINEAR_BACKWARD_BAD))])
def test_linear8_backward_refuses(kw, code):
    a = {"dy": BASE << 1, "x": BASE << 2, "dtype": 0, "rows": 40, "ld_dy": 5, "ld_x": 200, "wt": matrix(200, 5), "dx": BASE << 3, "ld_dx": 200,
         "dw": BASE << 4, "ld_dw": 200, "accumulate": False, "workspace": BASE << 5, "size": 0, **kw}
    need = c.mtdao_linear8_workspace_bytes(40, 5, 200)[1] + a.pop("size")
    with pytest.raises(abi.MtdaoError) as e:
        c.mtdao_linear8_backward(*a.values(), need, None)
    assert e.value.code == code


def test_linear8_sizes():
    assert c.mtdao_linear8_workspace_bytes(0, 5, 200)[0] == 0
    for sizes in ((-1, 5, 200), (5, -1, 200), (5, 5, -1), ((1 << 22) + 1, 5, 5), (5, (1 << 22) + 1, 5), (5, 5, (1 << 22) + 1)):
        with pytest.raises(abi.MtdaoError):
            c.mtdao_linear8_workspace_bytes(*sizes)
    c.mtdao_linear8(None, 0, 0, 200, matrix(5, 200), None, 0, 5, None, 0, None)


# ------------------------------------------------------------- torch level


def test_operators_refuse_cpu_tensors():
    x, w = torch.zeros(4, 64), torch.ones(64)
    for call in (lambda: ops.AdamW([x], [x]), lambda: ops.peri_norm(x, x, w, w), lambda: ops.peri_norm_backward(x, x, x, x, w, w),
                 lambda: ops.quantize8(x), lambda: ops.Weight8(x)):
        with pytest.raises(ValueError, match="GPU only"):
            call()


class Held:
    """A tensor as far as streams go."""

    device = torch.device("cuda", 0)

    def __init__(self):
        self.streams = []

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.streams.append(stream)


@pytest.fixture
def streams(monkeypatch):
    """streams[0]: the handle of the current stream."""
    now = [1]
    monkeypatch.setattr(ops, "_stream", lambda t: now[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: f"stream {now[0]}")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return now


@pytest.mark.parametrize("call", ["mtdao_adamw_step", "mtdao_adamw_set_grads"])
def test_adamw_keeps_what_it_allocated_for_the_streams_of_its_calls(call, streams, monkeypatch):
    seen = []
    monkeypatch.setattr(c, call, lambda *a: seen.append(a[-1]))
    opt = ops.AdamW.__new__(ops.AdamW)
    opt.handle, opt.params, opt._followed, opt.grads, opt.workspace = None, [], [], [torch.zeros(1)], Held()
    state = Held()
    opt._own, opt._streams = [opt.workspace, state], {1}
    monkeypatch.setattr(opt, "_grads_ok", lambda *a: None)
    go = (lambda: opt.step(0.1)) if call == "mtdao_adamw_step" else (lambda: opt.set_grads([]) or setattr(opt, "grads", [torch.zeros(1)]))
    for now in (1, 2, 2, 3, 1, 2):
        streams[0] = now
        go()
    assert seen == [1, 2, 2, 3, 1, 2]
    assert opt.workspace.streams == state.streams == ["stream 2", "stream 3"]


@pytest.mark.parametrize("call", ["mtdao_adamw_step", "mtdao_adamw_set_grads"])
def test_adamw_refuses_another_current_device(call, streams, monkeypatch):
    monkeypatch.setattr(c, call, lambda *a: pytest.fail("enqueued on another device"))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    opt = ops.AdamW.__new__(ops.AdamW)
    opt.handle, opt.params, opt.grads, opt.workspace, opt._own, opt._streams = None, [], [torch.zeros(1)], Held(), [], {1}
    monkeypatch.setattr(opt, "_grads_ok", lambda *a: None)
    with pytest.raises(ValueError, match="current device"):
        opt.step(0.1) if call == "mtdao_adamw_step" else opt.set_grads([])


def test_matrices_of_blocks_stay_for_the_streams_of_their_calls(streams, monkeypatch):
    seen = []
    for call in ("mtdao_quantize8", "mtdao_product8", "mtdao_linear8", "mtdao_linear8_backward"):
        monkeypatch.setattr(c, call, lambda *a: seen.append(a[-1]))
    monkeypatch.setattr(ops, "_on_device", lambda *a: torch.device("cpu"))

    def fake(rows, cols):
        q = ops.Matrix8(rows, cols, "cpu", ops.BLOCK)
        q._buf = Held()
        return q

    w = ops.Weight8.__new__(ops.Weight8)
    w.q, w.qt, a = fake(40, 256), fake(256, 40), fake(30, 256)
    x, y = torch.zeros(30, 256), torch.zeros(30, 40)
    for now, go, used in ((2, lambda: ops.linear8(x, w), [w.q]), (3, lambda: ops.linear8_backward(y, x, w), [w.qt]),
                          (4, lambda: w.update(torch.zeros(40, 256)), [w.q, w.qt]), (5, lambda: ops.product8(a, w.q, out=y), [a, w.q])):
        before = {m: list(m._buf.streams) for m in (w.q, w.qt, a)}
        for streams[0] in (1, now, now):
            go()
        for m, held in before.items():
            assert m._buf.streams == held + ([f"stream {now}"] if m in used else [])
    assert seen == [1, 2, 2, 1, 3, 3, 1, 4, 4, 1, 5, 5]


AT = 1 << 30  # from tensor to tensor in adamw_case


@pytest.mark.parametrize("kw", [dict(g__1=BASE), dict(g__0=BASE + 4), dict(g__0=BASE + AT + 3996), dict(g__2=BASE + AT + (2 << 26) - 3996),
                                dict(g__0=BASE + AT + (3 << 26)), dict(bits=8, g__0=BASE + (2 << 26)), dict(bits=8, g__1=BASE + (5 << 26)),
                                dict(bits=8, g__1=BASE + 2 * AT + (4 << 26) - 3996), dict(g__1=BASE, grad_dtype=1)], ids=str)
def test_adamw_refuses_gradients_on_what_it_writes(kw):
    cfg, rows = adamw_case(**kw)
    with pytest.raises(abi.MtdaoError, match="overlaps") as e:
        c.mtdao_adamw_init(cfg, rows, BASE << 1, 1 << 30, None)
    assert e.value.code == abi.MTDAO_ERR_INVALID_ARG


OUT_OF_MEMORY = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "host.hpp"
static bool none = false;
void* operator new(size_t n) {
  if (none) throw std::bad_alloc();
  return std::malloc(n);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }
int main() {
  std::string sink = "an earlier message";
  sink.shrink_to_fit();
  none = true;
  const int32_t code = mtdao::fail(&sink, MTDAO_ERR_WORKSPACE, "%s", "a message that does not fit into the string without more memory");
  none = false;
  std::printf("%d [%s]\n", code, sink.c_str());
}
"""


def test_errors_without_memory_for_their_message(tmp_path):
    """The code is returned; nothing is thrown through the C entry."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    src, exe = tmp_path / "oom.hip", tmp_path / "oom"
    src.write_text(OUT_OF_MEMORY)
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC", "-O3")]
    subprocess.run([build.HIPCC, *flags, "-O1", "-w", "-I", os.path.dirname(build.SRC), "-I", os.path.dirname(HEADER), "-o", str(exe), str(src)],
                   check=True, stderr=subprocess.DEVNULL)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert (r.returncode, r.stdout) == (0, f"{abi.MTDAO_ERR_WORKSPACE} []\n"), r
