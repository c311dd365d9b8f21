"""The bounds that the number format of the orthogonalised updates rests on (csrc/muon.hip), on
the CPU: two fp16 parts of a number, the singular values' polynomial, the exponents."""

import re

import torch

from lm_oracle import NS
from test_lm_ops_host import HEADER

A, B, C = NS


def test_two_halves_of_a_number():
    """x = hi + lo within 2^-23 |x|, which is reached; |lo| <= 2^-11 |x|, so lo lo <= 2^-22 of a product."""
    x = (1 + torch.rand(2_000_000, dtype=torch.float64, generator=torch.Generator().manual_seed(0))).float()
    x = torch.cat([x, torch.tensor([1 + 2 ** -11 - 2 ** -23, 1.0, 2 - 2 ** -23])])
    hi = x.half()
    lo = (x - hi.float()).half()
    off = ((x.double() - hi.double() - lo.double()) / x).abs()
    assert 2.0 ** -23.01 < float(off.max()) <= 2.0 ** -23
    assert 2.0 ** -24.6 < float(off.square().mean().sqrt()) < 2.0 ** -24.4
    assert float((lo.double() / x).abs().max()) <= 2.0 ** -11
    said = re.search(r"factors\s+\*?\s*in (\d+) bits", open(HEADER).read())
    assert said.group(1) == "23"


def test_singular_values_and_exponents():
    """Each stored factor fits fp16 with its exponent (14, 14, 13; 10 for what several steps make)."""
    s = torch.linspace(0, 1.21, 1_000_001, dtype=torch.float64)
    p = A * s + B * s ** 3 + C * s ** 5
    assert 1.2023 < float(p.max()) < 1.2024 and float(p.min()) >= 0
    g = s.square()
    poly = B * g + C * g * g
    assert float(poly.abs().max()) < 2.81 and float(g.max()) < 1.4642 and 1.2024 ** 2 < 1.46
    assert 0.63 < float((A + poly).min()) and float((A + poly).max()) <= A
    for most, exponent in ((1.21, 14), (1.46, 14), (2.81, 13), (A ** 3, 10)):
        assert most * 2.0 ** exponent < torch.finfo(torch.float16).max
