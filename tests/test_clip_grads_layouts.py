"""Lists of gradients whose rows lie anywhere: many short rows in long chunks, single rows with their values apart, tensors in the gaps of others."""
import ctypes
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import grads as gr

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


@gpu
@pytest.mark.parametrize("rows", [4000, 1_190_000])
def test_norm_of_many_short_rows(rows):
    """Rows of 131 values that do not start on 16 bytes, in chunks of 8192 and of 32 768 values.  The value's square is one whose fp32 sums are all rounded to the same side: 320 of them would be off by 80 u.

    A sum in fp32 has at most 34 values, two of them are added: 35 roundings of u, halved by the square root, and the result's: 18.5 u; counted as 20."""
    import torch
    value = 1.2773438
    g = torch.full((rows, 132), math.nan, dtype=torch.float16, device="cuda")[:, :131]
    g.fill_(value)
    v = float(g[0, 0])
    n = v * math.sqrt(rows * 131)
    assert abs(pkg.grad_norm([g]).item() - n) <= 20 * U * n


@gpu
def test_a_row_whose_values_lie_apart():
    """[1 x n] with a column stride, into a dense one and back."""
    import torch
    wide = torch.randn(1, 60, device="cuda")
    g, dense = wide[:, ::3], torch.randn(1, 20, device="cuda")
    n = math.sqrt(float((g.double() ** 2).sum()))
    out = torch.zeros(1, 20, device="cuda")
    pkg.clip_grads([g], n / 2, out=[out])
    assert bool(((out.double() - g.double() / 2).abs() <= 20 * U * g.double().abs()).all())
    keep = wide.clone()
    pkg.clip_grads([dense], math.inf, out=[wide[:, 1::3]])
    assert torch.equal(wide[:, 1::3], dense) and torch.equal(wide[:, ::3], keep[:, ::3]) and torch.equal(wide[:, 2::3], keep[:, 2::3])


def test_tensors_in_the_gaps_of_others():
    """On the host: what does not meet is let through (the call then lacks its workspace), what meets is refused."""
    L = gr._load()

    def call(*entries):
        return L.gad_clip_grads(gr._packer(len(entries)).pack(*[v for e in entries for v in e]), len(entries), 1.0, 256, None, 0, None)

    def part(row, col, rows, cols, ld):                         # of a matrix with 16 columns of fp32
        at = 4096 + 4 * (16 * row + col)
        return (at, 0, 0, rows, cols, ld, at, ld)
    left = part(0, 0, 8, 6, 16)
    for other in (part(3, 6, 1, 10, 16), part(3, 6, 1, 10, 10), part(0, 6, 1, 1, 1), part(1, 8, 3, 4, 32), part(0, 6, 4, 10, 48)):
        assert call(left, other) == -5 and call(other, left) == -5, other
    assert call(part(0, 0, 4, 16, 32), part(1, 3, 1, 9, 9)) == -5                               # every second row, and a piece of one between
    for other in (part(3, 5, 1, 3, 3), part(3, 6, 1, 11, 11), part(1, 8, 3, 9, 32), part(1, 5, 3, 4, 32), part(3, 0, 1, 1, 1), part(2, 8, 2, 4, 24), part(0, 3, 1, 40, 40)):
        assert call(left, other) == -1 and call(other, left) == -1, other
    assert call(part(0, 0, 4, 17, 32), part(1, 0, 1, 1, 1)) == -1 and call(part(0, 0, 4, 16, 32), part(2, 3, 1, 9, 9)) == -1
