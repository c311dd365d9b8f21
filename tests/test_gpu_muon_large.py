"""Orthogonalised updates (paper_2510_05361_amd.ops) of sizes that the products' larger tiles
take, against the definition in 64 bits on the GPU.  Padded to multiples of 128 the sides are
odd ones of it, so that the last tiles lie half outside, those on the diagonal too.  Which
kernels the cases reach is checked in test_lm_ops_instances.py.

Tolerance: a factor held in two fp16 parts is off by 2 U (U = 2^-24) where one of fp32 is by U at most, and what a
product leaves out, lo lo, is 4 U: 8 U a product at most where fp32's factors, rounded as they are
stored, make 2 U.  So four times what the same formulas in fp32 (torch on the GPU) are off by, or 64 U of the norm
as in test_gpu_muon.py; results are rounded once to their type."""

import pytest
import torch

import lm_oracle as oracle
from paper_2510_05361_amd import mtdao as abi
from paper_2510_05361_amd import mtdao_ops as c_ops
from paper_2510_05361_amd import ops

pytestmark = pytest.mark.gpu

U = oracle.U
DT = {"f32": torch.float32, "bf16": torch.bfloat16}

# batch, rows, cols: wide, tall, nearly square (a step at a time)
BIG = [(24, 1150, 1900), (24, 1900, 1150), (24, 1150, 1600)]
# one matrix whose squares are summed in chunks of several pieces
CHUNKS = [(1, 2900, 4400), (1, 4400, 2900)]
# more than 4 GiB of factors: a run of one shape in two groups
GROUPS = [(14, 2900, 4400)]
STEP = [(2900, 4400)] * 12 + [(4400, 2900), (1150, 1900), (300, 200), (64, 64)]


def matrices(shape, t, seed=0):
    return torch.empty(shape, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed)).to(DT[t])


def allowed(u64, u32, steps=5, eps=1e-7):
    """(result in 64 bits, norm of the error allowed) of a matrix."""
    want = oracle.newton_schulz(u64, steps, eps)
    off = (oracle.newton_schulz(u32, steps, eps).double() - want).norm()
    return want, max(4 * float(off), 64 * U * float(want.norm()))


def check(got, x):
    for i, (g, m) in enumerate(zip(got, x)):
        want, err = allowed(m.double(), m.float())
        err += oracle.half_step(got.dtype) * float(want.norm())
        off = float((g.double() - want).norm())
        assert off <= err, (i, off / err)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("batch,r,c", BIG)
def test_tiles_of_the_largest_size(batch, r, c, t):
    x = matrices((batch, r, c), t)
    x[5] = 0
    x[7, 3, 5] = float("nan")
    x[8, r - 1, c - 1] = float("inf")
    out = ops.orthogonalize(x)
    assert out.dtype == x.dtype and bool((out[5] == 0).all()) and bool(out[7:9].isnan().all())
    fine = [i for i in range(batch) if i not in (5, 7, 8)]
    check(out[fine], x[fine])
    assert torch.equal(ops.orthogonalize(x)[fine], out[fine])


@pytest.mark.parametrize("t,o", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("batch,r,c", CHUNKS)
def test_squares_of_large_matrices(batch, r, c, t, o):
    x = matrices((batch, r, c), t, 1)
    out = ops.orthogonalize(x, dtype=DT[o])
    check(out, x)
    assert torch.equal(ops.orthogonalize(x, dtype=DT[o]), out)


@pytest.mark.parametrize("batch,r,c", GROUPS)
def test_matrices_of_several_groups(batch, r, c):
    x = matrices((batch, r, c), "f32", 2)
    out = ops.orthogonalize(x)
    check(out, x)
    # the result in place of the matrices
    need = c_ops.mtdao_orthogonalize_workspace_bytes(batch, r, c)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    c_ops.mtdao_orthogonalize(x.data_ptr(), abi.MTDAO_F32, batch, r, c, x.data_ptr(), abi.MTDAO_F32, 5, 1e-7, ws.data_ptr(), need,
                              torch.cuda.current_stream().cuda_stream)
    assert torch.equal(x, out)


@pytest.mark.parametrize("p,g", [("f32", "bf16"), ("bf16", "f32")])
def test_steps_of_several_groups(p, g):
    params = [matrices(s, p, 10 + i).mul_(0.05) for i, s in enumerate(STEP)]
    grads = [matrices(s, g, 50 + i).mul_(0.01) for i, s in enumerate(STEP)]
    opt = ops.Muon(params, grads, weight_decay=0.1)
    lr, mu = 0.02, 0.95
    for _ in range(2):
        before = [[t.clone() for t in ts] for ts in (params, opt.m)]
        opt.step(lr)
        for i, (p0, m0, g0) in enumerate(zip(*before, grads)):
            r, c = p0.shape
            f = max(1.0, r / c) ** 0.5
            wm = mu * m0.double() + g0.double()
            assert bool(((opt.m[i].double() - wm).abs() <= 3 * U * (mu * m0.double().abs() + g0.double().abs()) + 1e-45).all()), i
            o, err = allowed(g0.double() + mu * wm, g0.float() + mu * (mu * m0 + g0.float()))
            want = p0.double() * (1 - lr * 0.1) - lr * f * o
            err = lr * f * err + 4 * U * float(p0.double().norm()) + oracle.half_step(p0.dtype) * float(want.norm())
            off = float((params[i].double() - want).norm())
            assert off <= err, (i, off / err)
