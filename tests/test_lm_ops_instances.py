"""Which kernels, with which template arguments, the GPU tests of the orthogonalised updates, the
embedding and the cross entropy reach: every one that the library has (CPU: launches are taken
down, nothing runs), so that a rule on sizes that moves drops none from the tests unseen."""

import re
import subprocess

import pytest

import launch_recorder
import test_gpu_cross_entropy
import test_gpu_cross_entropy_widths
import test_gpu_embedding
import test_gpu_muon
import test_gpu_muon_large
from paper_2510_05361_amd import build


@pytest.fixture(scope="module")
def instances(tmp_path_factory):
    shim = launch_recorder.build(str(tmp_path_factory.mktemp("shim")))
    return lambda body: launch_recorder.instances(shim, body)


def in_the_library(prefix):
    """The kernels whose names begin so, with their arguments, from the host's symbols."""
    out = subprocess.run(["nm", "-C", build.LIB], capture_output=True, text=True, check=True).stdout
    found = re.findall(r"__device_stub__(" + prefix + r"\w*(?:<[^(]*>)?)\(", out)
    return {f.replace("unsigned short", "bf16") for f in found}


def cases_of(test, names):
    """The values that a test is run with."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)


ORTHOGONALIZE = """
        B = 1 << 40
        for batch, r, k in {cases}:
            for t in (0, 1):
                need = c.mtdao_orthogonalize_workspace_bytes(batch, r, k)
                c.mtdao_orthogonalize(B, t, batch, r, k, B << 8, {out}, 5, 1e-7, B << 16, need, None)
"""
MUON = """
        B = 1 << 40
        shapes = {shapes}
        rows = (c.MuonMatrix * len(shapes))(*(c.MuonMatrix(*(B + (i << 46) + (j << 43) for j in range(3)), *s, 0.1, 1.0) for i, s in enumerate(shapes)))
        for p, g in {types}:
            cfg = c.MuonConfig(p, g, len(shapes), 1, 5, 0, 0.9, 1e-7)
            h = c.mtdao_muon_init(cfg, rows, B << 20, c.mtdao_muon_workspace_bytes(cfg, rows), None)
            c.mtdao_muon_step(h, 1e-3, None)
            c.mtdao_muon_destroy(h)
"""


def products(names):
    return {n for n in names if n.startswith("k_muon_product")}


@pytest.mark.parametrize("batch,r,c", test_gpu_muon_large.BIG)
def test_large_batches_are_multiplied_in_the_largest_tiles(instances, batch, r, c):
    names = instances(ORTHOGONALIZE.format(cases=[(batch, r, c)], out="t"))
    assert products(names) == {"k_muon_product<256, 2, 4, 2, float>", "k_muon_product<256, 2, 4, 2, bf16>"}


def test_groups_and_chunks(instances):
    """A launch of sums for each group; squares of large matrices in several pieces a chunk."""
    for cases in (test_gpu_muon_large.GROUPS,):
        names = instances(ORTHOGONALIZE.format(cases=cases, out="t"))
        assert names.count("k_muon_sums<float, false>") == 2 and "k_muon_product<256, 2, 4, 2, float>" in names
    names = instances(MUON.format(shapes=test_gpu_muon_large.STEP, types=[(0, 1)]))
    assert names.count("k_muon_sums<bf16, true>") == 2 and {"k_muon_tiny<bf16, float, true, 2>"} < set(names)
    assert {"k_muon_product<256, 2, 4, 2, float>", "k_muon_product<128, 2, 2, 2, float>"} <= products(names)
    assert all(r * k > 4096 * 1024 for _, r, k in test_gpu_muon_large.CHUNKS)  # pieces of a chunk, chunks of a matrix


def test_every_kernel_of_the_updates(instances):
    """The sizes of the tests, in their pairs of types."""
    one = [(1, r, c) for r, c in cases_of(test_gpu_muon.test_sizes, "r,c")]
    seen = instances(ORTHOGONALIZE.format(cases=one + test_gpu_muon_large.BIG + test_gpu_muon_large.GROUPS, out="t"))
    seen += instances(ORTHOGONALIZE.format(cases=[(6, 90, 50), (6, 20, 50)], out="1 - t"))
    seen += instances(ORTHOGONALIZE.format(cases=test_gpu_muon_large.CHUNKS, out="0"))
    seen += instances(MUON.format(shapes=test_gpu_muon.MODEL + [(5, 3), (1, 1), (300, 7), (130, 129), (20, 30)], types=[(p, g) for p in (0, 1) for g in (0, 1)]))
    seen += instances(MUON.format(shapes=[(20, 30)], types=[(p, g) for p in (0, 1) for g in (0, 1)]))
    seen += instances(MUON.format(shapes=test_gpu_muon_large.STEP, types=[(0, 1), (1, 0)]))
    assert set(seen) == in_the_library("k_muon")


@pytest.mark.parametrize("cols", [9000, 32003, 50304])
def test_rows_that_share_cus_have_fewer_threads(instances, cols):
    """1024 threads a row while each row has a CU, 256 where they share them."""
    for rows, threads in ((1, 1024), (256, 1024), (257, 256), (384, 256), (4096, 256)):
        names = instances(f"""
        B = 1 << 40
        a = c.CrossEntropyArgs({rows}, {cols}, {cols}, {cols}, 1, 64, 0, 0.0, 1.0, 0, B, B << 14, None, B << 16, None, None)
        c.mtdao_cross_entropy(a, B << 20, 0, None)
        """)
        assert names == [f"k_cross_entropy<bf16, {threads}>"], (rows, names)


def test_every_kernel_of_the_cross_entropy(instances):
    cases = [(r, c, d) for r, c in test_gpu_cross_entropy.SIZES for d in (0, 1)] + [(7, c, d) for c in test_gpu_cross_entropy_widths.HELD for d in (0, 1)]
    cases += [(r, c, 0) for r, c in test_gpu_cross_entropy_widths.EVALUATION]
    seen = instances(f"""
        B = 1 << 40
        for rows, cols, gradient in {cases}:
            for t in (0, 1):
                a = c.CrossEntropyArgs(rows, cols, cols, cols, t, 64, 2, 0.0, 1.0, 0, B, B << 14, None, None, B << 16, (B << 18) if gradient else None)
                c.mtdao_cross_entropy(a, B << 20, c.mtdao_cross_entropy_workspace_bytes(a), None)
    """)
    assert set(seen) == in_the_library("k_cross_entropy")
    assert {"k_cross_entropy<float, 256>", "k_cross_entropy<bf16, 256>"} <= set(seen)


def test_many_places_are_sorted_in_tiles(instances):
    """Passes in which every workgroup counts all places take longer than tiles from some 16384 places on."""
    for n, kernel in ((2049, "k_embedding_pass<8>"), (16384, "k_embedding_pass<8>"), (16385, "k_embedding_move"), (65536, "k_embedding_move")):
        names = instances(f"""
        B = 1 << 40
        need = c.mtdao_embedding_backward_workspace_bytes({n}, 50304, 64)
        c.mtdao_embedding_backward(B << 14, 0, 64, B, 64, {n}, 1.0, B << 16, 50304, 64, 64, 0, B << 18, need, None)
        """)
        sorts = {x for x in names if re.match("k_embedding_(sort|pass|move)", x)}
        assert sorts == {kernel}, (n, names)


def test_every_kernel_of_the_embedding(instances):
    rows = cases_of(test_gpu_embedding.test_lookup, "n,rows,d")
    sums = cases_of(test_gpu_embedding.test_sums, "n,rows,d")
    seen = instances(f"""
        B = 1 << 40
        for n, rows, d in {rows}:
            for w in (0, 1):
                for y in (0, 1):
                    c.mtdao_embedding(B, 64, n, B << 14, w, rows, d, d, 1.0, B << 16, y, d, None)
        for n, rows, d in {sums}:
            for t in (0, 1):
                for onto in (0, 1):
                    need = c.mtdao_embedding_backward_workspace_bytes(n, rows, d)
                    c.mtdao_embedding_backward(B << 14, t, d, B, 64, n, 1.0, B << 16, rows, d, d, onto, B << 18, need, None)
    """)
    assert set(seen) == in_the_library("k_embedding")
