"""Where the gated feed-forward block could lose more than its results' own rounding, or hide what is no number: long sums of few rows, gelu's tail, infinite values.

u = 2^-24.  What is promised of 16-bit types is that the tensor core adds up no more than a chunk (fp16 8192 terms, bfloat16 65 536) before the sum goes on in fp32, each 16 terms cut off by at most 2 u of it:
an eighth of the results' rounding, counted here with a rounding of fp32 a chunk and share.  The cuts are all to one side, so they show in the mean, where the results' own roundings (uniform where
results spread over steps of their type, of standard deviation eps / 2 / sqrt 3 at most) leave six of theirs over the square root of the number of results."""
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def positive(rows, cols, g, dtype):
    import torch
    return torch.rand(rows, cols, generator=g, device="cuda").add_(0.5).to(dtype)


def one_column(rows, cols, dtype, values=1.0):
    """A matrix with values in its first column, and nothing else."""
    import torch
    m = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    m[:, 0] = values
    return m


def cut_off(K, chunk):
    """Of a sum of K positive products: the tensor core's cuts (and up to 8 for the sums of 16 themselves), a rounding a chunk and share, at most 64 of these."""
    return 2 * U * (min(K, chunk) / 16 + 8) + U * (K / chunk + 64)


def held(got, want, K, chunk):
    import torch
    half = torch.finfo(got.dtype).eps / 2
    off = got.double() / want - 1
    assert float(off.abs().max()) <= (1 + 2 * half) * half + cut_off(K, chunk)
    # Positive terms of sum 1 and their K factors in 0.5 .. 1.5: results spread by 0.3 / sqrt K.  fp16: 1.4e-3 and 1.9e-3, two to four steps of at most 2^-10; bfloat16: 0.8e-3, a tenth of a step of
    # 2^-7, so that all are rounded alike and their mean is no measure.
    if got.dtype != torch.float16:
        return
    assert abs(float(off.mean())) <= 6 * half / math.sqrt(3 * off[:1].numel()) + cut_off(K, chunk), float(off.mean())


@gpu
@pytest.mark.parametrize("rows", [1, 16, 200, 300])
def test_long_sums_of_few_rows(rows):
    """In the forms for up to 256 rows, and in tiles.  Sums of one sign, which lose most.  First y: g is one value a unit and u is 1, so h is exact and the down projection alone rounds.  Then h: a down projection that hands it on."""
    import torch
    dt, chunk = torch.float16, 8192
    g = torch.Generator(device="cuda").manual_seed(rows)
    D, F = 8192, 49_152
    a = (torch.rand(F, generator=g, device="cuda") + 0.5).to(dt)
    x, Wd = one_column(rows, D, dt), positive(D, F, g, dt).div_(16)
    y = pkg.gated_feed_forward(x, one_column(F, D, dt, a), one_column(F, D, dt), Wd, activation="relu").check().y
    held(y, (Wd.double() @ a.double())[None].expand(rows, D), F, chunk)

    D, F = 24_576, 8192
    x, Wg = positive(rows, D, g, dt), positive(F, D, g, dt).div_(16)
    x[:, 0] = 1
    y = pkg.gated_feed_forward(x, Wg, one_column(F, D, dt), torch.eye(D, F, dtype=dt, device="cuda"), activation="relu").check().y
    held(y[:, :F], x.double() @ Wg.double().t(), D, chunk)
    assert not y[:, F:].any()


@gpu
def test_long_sums_of_a_weights_gradient():
    """Over 50 000 rows, in whole tiles."""
    import torch
    dt, N, D, F = torch.float16, 50_000, 2304, 2304
    g = torch.Generator(device="cuda").manual_seed(7)
    dy, h = positive(N, D, g, dt).div_(16), positive(N, F, g, dt)
    W = torch.zeros(F, D, dtype=dt, device="cuda")
    got = pkg.gated_feed_forward_backward(dy, dy, W, W, W, h, h, h, grads="d").check().dWd
    held(got, dy.double().t() @ h.double(), N, 8192)


@gpu
def test_long_sums_of_few_rows_in_bfloat16():
    """A bfloat16 chunk has 65 536 terms; a reduction of two of them and a rest, with enough tiles that it is not cut into shares that short."""
    import torch
    dt = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(5)
    D, F = 9472, 140_000
    a = (torch.rand(F, generator=g, device="cuda") + 0.5).to(dt)
    Wd = positive(D, F, g, dt).div_(1 << 17)
    y = pkg.gated_feed_forward(one_column(3, D, dt), one_column(F, D, dt, a), one_column(F, D, dt), Wd, activation="relu").check().y
    held(y, torch.stack([Wd[i:i + 1184].double() @ a.double() for i in range(0, D, 1184)]).reshape(1, D).expand(3, D), F, 65_536)


def test_half_of_log2_e_in_two_parts():
    """exp(-x^2 / 2) takes x^2 log2(e) / 2 with more than fp32's bits: the constant's two parts together are off by no more than the second's rounding."""
    import os
    import re
    import numpy as np
    text = open(os.path.join(os.path.dirname(pkg.__file__), "csrc", "gated_gemm.cuh")).read()
    c, lo = (float(np.float32(v)) for v in re.search(r"exp_half_square.*?c = ([0-9.e-]+)f, c_lo = ([0-9.e-]+)f", text, re.S).groups())
    assert abs(c + lo - math.log2(math.e) / 2) <= 1e-4 * abs(lo)


@gpu
def test_gelus_tail():
    """fp32: the error relative to gelu itself does not grow with |g|.

    u a part: the fit 2; t 5 (a quotient of 2 ulp, a rounding), which count 1 + 1.3 t times; the exponent's polynomial 4 and its scaling 1.5; two exponentials 3 each; products 4.  On average the roundings go (4000
    values of either sign), and what may stay is the fit's 2, an ulp of each exponential and of the quotient, and 1 for the rest: 10."""
    import torch
    for lo, hi in ((-12.9, -12.4), (-12.9, -6.0), (-6.0, -1.0), (-1.0, -1e-3), (1e-3, 13.0)):
        x = torch.linspace(lo, hi, 4001, device="cuda")[:, None]
        one = torch.ones(1, 1, device="cuda")
        act = pkg.gated_feed_forward(x, one, one, one, activation="gelu", save=True).check().act
        z = -x.double() / math.sqrt(2)
        rel = act.double() / (x.double() * 0.5 * torch.erfc(z)) - 1
        t = 1 / (1 + 0.5 * z.abs())
        bound = (2 + 5 * (1 + 1.3 * t) + 4 + 1.5 + 6 + 4) * U
        assert bool((rel.abs() <= bound).all()), (lo, hi, float((rel.abs() - bound).max()) / U)
        assert abs(float(rel.mean())) <= 10 * U, (lo, hi, float(rel.mean()) / U)


@gpu
@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu", "sigmoid"])
def test_infinite_gates(kind, rows):
    """g of -infinity and infinity beside a finite u: what the formulas give, in the forms for few rows and in tiles.  silu and gelu of -infinity are 0 times infinity, no number."""
    import torch
    x = torch.ones(rows, 1, dtype=torch.float64, device="cuda")
    x[::2] = -1
    g = x * math.inf
    if kind == "relu":
        a, d = g.clamp(min=0), (g > 0).double()
    elif kind == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        a, d = g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        s = 1 / (1 + torch.exp(-g))
        a, d = (s, s * (1 - s)) if kind == "sigmoid" else (g * s, s * (1 + g * (1 - s)))
    want = dict(act=a, slope=x * d, h=a * x, y=a * x)
    for dtype in (torch.bfloat16, torch.float16) + ((torch.float32,) if rows <= 16 else ()):
        one = torch.ones(1, 1, dtype=dtype, device="cuda")
        for save in (False, True) if dtype != torch.float32 else (False,):
            r = pkg.gated_feed_forward(x.to(dtype), one * math.inf, one, one, activation=kind, save=save).check()
            for name, w in want.items():
                t = getattr(r, name)
                if t is not None:
                    assert torch.equal(t.double().nan_to_num(nan=7.0), w.nan_to_num(nan=7.0)), (name, dtype, save)


@gpu
@pytest.mark.parametrize("rows", [6, 40])
def test_infinite_values_in_fp32(rows):
    """Up to 16 rows as the formulas have them; where operands are taken in three parts, no numbers in all that they have a part in, and in nothing else."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    D, F = 72, 136
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, Wg, Wu, Wd, dy = r(rows, D), r(F, D) / 8, r(F, D) / 8, r(D, F) / 8, r(rows, D)
    clean = pkg.gated_feed_forward(x, Wg, Wu, Wd, activation="sigmoid").y
    saved = pkg.gated_feed_forward(x, Wg, Wu, Wd, activation="sigmoid", save=True)
    others = torch.arange(rows, device="cuda") != 3
    columns = torch.arange(D, device="cuda") != 5

    xi, Wi = x.clone(), Wd.clone()
    xi[3, 7], Wi[5, 9] = math.inf, -math.inf
    y = pkg.gated_feed_forward(xi, Wg, Wu, Wd, activation="sigmoid").check().y
    want = (torch.sigmoid(xi[3:4].double() @ Wg.double().t()) * (xi[3:4].double() @ Wu.double().t())) @ Wd.double().t()
    assert torch.equal(y[others], clean[others]) and not bool(y[3].isfinite().any()) and (rows <= 16 or bool(y[3].isnan().all())) and not bool(want.isfinite().any())
    y = pkg.gated_feed_forward(x, Wg, Wu, Wi, activation="sigmoid").check().y
    want = -math.inf * saved.h[:, 9]
    assert torch.equal(y[:, columns], clean[:, columns]) and (torch.equal(y[:, 5], want) if rows <= 16 else bool(y[:, 5].isnan().all()))
    kept = pkg.gated_feed_forward(xi, Wg, Wu, Wd, activation="sigmoid", save=True).check()
    assert all(bool(getattr(kept, k)[3].isnan().all()) and torch.equal(getattr(kept, k)[others], getattr(saved, k)[others]) for k in ("y", "act", "slope", "h"))
    dyi = dy.clone()
    dyi[3, 7] = math.inf
    b = pkg.gated_feed_forward_backward(dyi, x, Wg, Wu, Wd, saved.act, saved.slope, saved.h).check()
    assert bool(b.dx[3].isnan().all()) and bool(b.dx[others].isfinite().all())
    assert bool(b.dWd[7].isnan().all()) and bool(b.dWd[torch.arange(D, device="cuda") != 7].isfinite().all())
