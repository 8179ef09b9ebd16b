"""Gated feed-forward block and its backward pass against the formulas in 64 bits.

Tolerances, element by element and with a factor of 1.  u = 2^-24.  A sum of K products is off by at most ``steps(K)`` 2u times the sum of their magnitudes: the tensor core adds 16 products at
a time and cuts off at most 2u of the accumulator each time (fp32 operands in three parts: six sums, five of them 2^-8 of the first, and 2^-24 dropped; counted as K / 16 + K / 256 + 16 steps).
act and its slope come from exp2 (or erfc) and a reciprocal: (8 + 2 |g|) u relative for act, four times that, absolutely, for the slope (its values are below 1.2); |act'| < 1.2 and |act''| < 1 carry g's error on (relu's
slope jumps: where |g| is within its error of zero the slope may be either).  What is rounded to 16 bits is off by half a step, eps / 2 of its value, or of fp16's smallest normal."""
import ctypes
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import GadError
from paper_2110_02987_b200 import feed_forward as ff

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def steps(K, dtype):
    import torch
    return 2 * U * (K / 16 + K / 256 + 16 if dtype == torch.float32 else K / 16 + 8)


def half(v, dtype):
    """Half a step of dtype at v."""
    import torch
    f = torch.finfo(dtype)
    return f.eps / 2 * v.abs().clamp(min=f.tiny)


def matrix(rows, cols, dtype, g, scale=1.0, pad=0, offset=0):
    import torch
    m = torch.randn(rows, cols, generator=g, dtype=torch.float64) * scale
    buf = torch.full((rows * (cols + pad) + offset,), math.nan, dtype=dtype, device="cuda")     # what lies between the rows is no number
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(m)
    return v


def make(N, D, F, dtype, seed=0, pad=0, offset=0, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)
    return dict(x=matrix(N, D, dt, g, scale, pad, offset), Wg=matrix(F, D, dt, g, 1 / math.sqrt(D), pad, offset), Wu=matrix(F, D, dt, g, 1 / math.sqrt(D), pad, offset),
                Wd=matrix(D, F, dt, g, 1 / math.sqrt(F), pad, offset))


def activation(kind, g):
    import torch
    if kind == "relu":
        return g.clamp(min=0), (g > 0).double()
    if kind == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if kind == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def forward(x, Wg, Wu, Wd, kind):
    """(values, tolerances) of y, act, slope and h."""
    dt, D, F = x.dtype, x.shape[1], Wg.shape[0]
    x, Wg, Wu, Wd = (t.double() for t in (x, Wg, Wu, Wd))
    g, u = x @ Wg.t(), x @ Wu.t()
    eg, eu = (steps(D, dt) * (x.abs() @ w.abs().t()) for w in (Wg, Wu))
    a, d = activation(kind, g)
    rel = (8 + 2 * g.abs()) * U
    ea, ed = 1.2 * eg + rel * a.abs(), eg + 4 * rel
    if kind == "relu":
        ed = (g.abs() <= eg).double()
    h, s = a * u, u * d
    eh = a.abs() * eu + u.abs() * ea + ea * eu + half(h, dt)
    y = h @ Wd.t()
    ey = eh @ Wd.abs().t() + steps(F, dt) * ((h.abs() + eh) @ Wd.abs().t()) + half(y, dt)
    return dict(y=(y, ey), act=(a, ea + half(a, dt)), slope=(s, (d.abs() + ed) * eu + u.abs() * ed + half(s, dt)), h=(h, eh))


def backward(dy, x, Wg, Wu, Wd, act, slope, h):
    dt, N, D, F = x.dtype, x.shape[0], x.shape[1], Wg.shape[0]
    dy, x, Wg, Wu, Wd, act, slope, h = (t.double() for t in (dy, x, Wg, Wu, Wd, act, slope, h))
    dh, eh = dy @ Wd, steps(D, dt) * (dy.abs() @ Wd.abs())
    dg, du = dh * slope, dh * act
    eg, eu = slope.abs() * eh + half(dg, dt), act.abs() * eh + half(du, dt)
    dx = dg @ Wg + du @ Wu
    ex = eg @ Wg.abs() + eu @ Wu.abs() + steps(2 * F, dt) * ((dg.abs() + eg) @ Wg.abs() + (du.abs() + eu) @ Wu.abs())
    out = dict(dx=(dx, ex + half(dx, dt)))
    for name, m, e, v in (("dWg", dg, eg, x), ("dWu", du, eu, x), ("dWd", dy, 0 * dy, h)):
        w = m.t() @ v
        out[name] = w, e.t() @ v.abs() + steps(N, dt) * ((m.abs() + e).t() @ v.abs()) + half(w, dt)
    return out


def near(got, want):
    import torch
    for name, (v, tol) in want.items():
        t = getattr(got, name)
        assert t.shape == v.shape, name
        # the final rounding is of what was computed, which may lie a step higher
        off = (t.double() - v).abs() - tol * (1 + torch.finfo(t.dtype).eps)
        assert bool((off <= 1e-30).all()), "%s: %g over its tolerance, %d of %d" % (name, float(off.max()), int((~(off <= 1e-30)).sum()), off.numel())


SIZES = [(1, 1, 1), (2, 3, 5), (1, 64, 128), (3, 200, 72), (5, 57, 33), (16, 128, 256), (17, 129, 257), (48, 256, 640), (128, 64, 129), (129, 200, 127), (256, 256, 256), (257, 500, 300), (300, 1433, 77),
         (1000, 72, 1433), (64, 128, 5000), (2500, 320, 640)]


@gpu
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,D,F", SIZES)
def test_forward_and_backward(N, D, F, dtype):
    i = SIZES.index((N, D, F))
    kind = ("silu", "gelu", "relu", "sigmoid")[i % 4]
    pad, offset = ((0, 0), (5, 3), (8, 0))[i % 3]
    s = make(N, D, F, dtype, i, pad, offset)
    r = pkg.gated_feed_forward(**s, activation=kind, save=True).check()
    near(r, forward(**s, kind=kind))
    plain = pkg.gated_feed_forward(**s, activation=kind).check()
    assert plain.act is None and plain.slope is None and plain.h is None
    near(plain, {"y": forward(**s, kind=kind)["y"]})
    import torch
    dy = matrix(N, D, s["x"].dtype, torch.Generator().manual_seed(100 + i), 0.5, pad, offset)
    near(pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h).check(), backward(dy, **s, act=r.act, slope=r.slope, h=r.h))


@gpu
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,D,F", [(1, 2048, 8192), (2, 999, 2050), (3, 4100, 130), (4, 64, 20_000), (5, 131, 77), (7, 2000, 13_000), (16, 300, 1000), (17, 300, 1000), (31, 4096, 64), (64, 520, 3000),
                                   (100, 72, 5000), (255, 640, 1000), (256, 1000, 640)])
def test_serving(N, D, F, dtype):
    """Nothing kept: the forms for few rows, their cuts, rows that do not start on 16 bytes."""
    kind = ("silu", "gelu", "relu", "sigmoid")[N % 4]
    for pad, offset in ((0, 0), (4, 1)):
        s = make(N, D, F, dtype, N, pad, offset)
        r = pkg.gated_feed_forward(**s, activation=kind).check()
        near(r, {"y": forward(**s, kind=kind)["y"]})
        again = pkg.gated_feed_forward(**s, activation=kind).check()
        import torch
        assert torch.equal(r.y, again.y)


@gpu
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu", "sigmoid"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_activations_over_their_range(kind, dtype):
    """One column: g and u are x itself, from 0 to where the exponentials under- and overflow."""
    import torch
    v = torch.cat([torch.linspace(-12, 12, 401), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 40.0, -40.0, 87.0, -87.0, 89.0, -89.0, 110.0, -110.0, 3e4, -3e4, 1e18, -1e18])])
    x = v.to(getattr(torch, dtype)).cuda()[:, None]
    one = torch.ones(1, 1, dtype=x.dtype, device="cuda")
    r = pkg.gated_feed_forward(x, one, one, one, activation=kind, save=True).check()
    want = forward(x, one, one, one, kind)
    # where act is below the smallest normal numbers it may be zero
    tiny = 2.0 ** -125
    near(r, {k: (v, t + tiny * (1 + x.double().abs())) for k, (v, t) in want.items()})
    assert all(bool(t.isfinite().all()) for t in (r.act, r.slope))


@gpu
def test_no_number_stays_in_its_row():
    import torch
    s = make(300, 96, 200, "bfloat16", 3)
    want = pkg.gated_feed_forward(**s, save=True)
    s["x"][7, 5] = math.nan
    s["x"][290, 0] = math.inf
    for kind in ("silu", "gelu", "relu", "sigmoid"):
        r = pkg.gated_feed_forward(**s, activation=kind, save=True).check()
        rows = torch.ones(300, dtype=torch.bool, device="cuda")
        rows[7] = rows[290] = False
        assert bool(r.y[7].isnan().all())
        if kind == "silu":
            assert all(torch.equal(getattr(r, k)[rows], getattr(want, k)[rows]) for k in ("y", "act", "slope", "h"))


@gpu
@pytest.mark.parametrize("N,D,F,dtype", [(8300, 256, 9472, "float16"), (700, 8300, 2304, "float16"), (9000, 256, 256, "bfloat16")])
def test_long_sums(N, D, F, dtype):
    """Reductions of more than a chunk in tiles that are not cut, and cut ones; sums of one sign, which lose most."""
    import torch
    s = make(N, D, F, dtype, 5, scale=0.2)
    for k in ("x", "Wg", "Wu", "Wd"):
        s[k] = s[k].abs()
    r = pkg.gated_feed_forward(**s, save=True).check()
    near(r, forward(**s, kind="silu"))
    dy = matrix(N, D, s["x"].dtype, torch.Generator().manual_seed(6), 0.01).abs()
    near(pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h).check(), backward(dy, **s, act=r.act, slope=r.slope, h=r.h))


@gpu
def test_offsets_behind_32_bits():
    """More than 2^31 units in all: the last rows, and the gradients' sums over all of them, against the same call on pieces."""
    import torch
    N, D, F = 70_000, 64, 32_768
    g = torch.Generator(device="cuda").manual_seed(40)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy = r(N, D).bfloat16(), (0.01 * r(N, D)).bfloat16()
    W = (r(F, D) / 8).bfloat16(), (r(F, D) / 8).bfloat16(), (r(D, F) / 180).bfloat16()
    f = pkg.gated_feed_forward(x, *W, save=True).check()
    b = pkg.gated_feed_forward_backward(dy, x, *W, f.act, f.slope, f.h).check()
    parts = [0.0, 0.0, 0.0]
    for i in range(0, N, 10_000):
        j = slice(i, i + 10_000)
        p = pkg.gated_feed_forward(x[j], *W, save=True)
        assert all(torch.equal(getattr(p, k), getattr(f, k)[j]) for k in ("act", "slope", "h"))
        q = pkg.gated_feed_forward_backward(dy[j], x[j], *W, p.act, p.slope, p.h)
        # (how sums are cut goes by the sizes: one rounding on either side)
        for u, v in ((p.y, f.y[j]), (q.dx, b.dx[j])):
            assert float((u.double() - v.double()).norm()) <= 2.0 ** -8 * float(v.double().norm())
        for k, t in enumerate((q.dWg, q.dWu, q.dWd)):
            parts[k] = parts[k] + t.double()
    for t, want in zip((b.dWg, b.dWu, b.dWd), parts):     # seven parts, each rounded, and the whole
        assert float((t.double() - want).norm()) <= 2.0 ** -8 * math.sqrt(8) * float(want.norm())


@gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_some_of_the_gradients(dtype):
    import torch
    s = make(200, 136, 264, dtype, 8)
    r = pkg.gated_feed_forward(**s, save=True)
    dy = matrix(200, 136, s["x"].dtype, torch.Generator().manual_seed(9))
    exact = backward(dy, **s, act=r.act, slope=r.slope, h=r.h)
    names = {"x": "dx", "g": "dWg", "u": "dWu", "d": "dWd"}
    # (how sums are cut into shares goes by what is asked for: each is within the tolerance, not the same to the bit)
    for want in ("x", "g", "u", "d", "xd", "gu", "ud", ""):
        some = pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h, grads=want).check()
        assert all(getattr(some, name) is None for k, name in names.items() if k not in want)
        near(some, {names[k]: exact[names[k]] for k in want})


@gpu
def test_gradients_against_differences():
    """Along random directions of x and of every weight: central differences of sum(y dy) in 64 bits (off by 1e-7 of it at a step of 1e-4)."""
    import torch
    s = make(60, 40, 72, "float32", 11)
    g = torch.Generator().manual_seed(12)
    dy = matrix(60, 40, torch.float32, g)
    for kind in ("silu", "gelu", "sigmoid"):
        r = pkg.gated_feed_forward(**s, activation=kind, save=True)
        b = pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h).check()
        for k, name in (("x", "dx"), ("Wg", "dWg"), ("Wu", "dWu"), ("Wd", "dWd")):
            v = torch.randn(s[k].shape, generator=g, dtype=torch.float64).cuda()
            at = []
            for e in (1e-4, -1e-4):
                p = {n: t.double() + e * v if n == k else t.double() for n, t in s.items()}
                a, _ = activation(kind, p["x"] @ p["Wg"].t())
                at.append(float(((a * (p["x"] @ p["Wu"].t())) @ p["Wd"].t() * dy.double()).sum()))
            want = (at[0] - at[1]) / 2e-4
            got, size = float((getattr(b, name).double() * v).sum()), float((getattr(b, name).double() * v).abs().sum())
            assert abs(got - want) <= 2e-6 * size, (kind, k, got, want)


@gpu
def test_rows_that_are_one_row():
    import torch
    s = make(40, 64, 96, "float16", 14)
    s["x"] = s["x"][:1].expand(40, 64)
    r = pkg.gated_feed_forward(**s, save=True).check()
    near(r, forward(**s, kind="silu"))
    dy = matrix(1, 64, torch.float16, torch.Generator().manual_seed(15)).expand(40, 64)
    near(pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h).check(), backward(dy, **s, act=r.act, slope=r.slope, h=r.h))


@gpu
def test_saved_tensors_of_any_layout():
    import torch
    s = make(70, 48, 77, "bfloat16", 16)
    r = pkg.gated_feed_forward(**s, save=True)
    dy = matrix(70, 48, torch.bfloat16, torch.Generator().manual_seed(17))
    want = pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h)
    got = pkg.gated_feed_forward_backward(dy, **s, act=r.act.contiguous(), slope=r.slope.contiguous(), h=r.h.contiguous())
    assert all(torch.equal(u, v) for u, v in zip(got, want))


@gpu
def test_equal_calls_streams_and_graphs():
    import torch
    s = make(500, 192, 320, "bfloat16", 20)
    dy = matrix(500, 192, torch.bfloat16, torch.Generator().manual_seed(21))

    def step(stream=None):
        r = pkg.gated_feed_forward(**s, save=True, stream=stream)
        return tuple(r) + tuple(pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h, stream=stream))
    want = step()
    assert all(torch.equal(u, v) for u, v in zip(step(), want))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [step(t) for t in streams * 3]                                    # two at once
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for got in both for u, v in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for t in out:
        t.fill_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(out, want))


@gpu
@pytest.mark.parametrize("N,D,F", [(257, 512, 320), (100, 500, 128), (300, 700, 1440)])
def test_calls_whose_tiles_go_to_slots_give_equal_bits(N, D, F):
    """Few tiles of fp32: what a warp reads back of its sums is its own."""
    import torch
    s = make(N, D, F, "float32", 30)
    dy = matrix(N, D, torch.float32, torch.Generator().manual_seed(31))
    want = None
    for _ in range(30):
        r = pkg.gated_feed_forward(**s, save=True)
        got = tuple(r) + tuple(pkg.gated_feed_forward_backward(dy, **s, act=r.act, slope=r.slope, h=r.h))
        want = want or got
        assert all(torch.equal(u, v) for u, v in zip(got, want))


@gpu
def test_no_rows():
    import torch
    W, Wd = torch.ones(10, 16, device="cuda"), torch.ones(16, 10, device="cuda")
    r = pkg.gated_feed_forward(torch.empty(0, 16, device="cuda"), W, W, Wd, save=True).check()
    assert r.y.shape == (0, 16) and r.h.shape == (0, 10)
    b = pkg.gated_feed_forward_backward(r.y, r.y, W, W, Wd, r.act, r.slope, r.h).check()
    assert b.dx.shape == (0, 16) and not b.dWg.any() and not b.dWu.any() and not b.dWd.any()


@gpu
def test_refusals_of_tensors():
    import torch
    s = make(6, 16, 24, "float32", 1)
    r = pkg.gated_feed_forward(**s, save=True)
    saved = dict(act=r.act, slope=r.slope, h=r.h)
    dy = torch.ones(6, 16, device="cuda")
    for change in (dict(Wg=s["Wg"].half()), dict(Wg=s["Wg"][:, :8]), dict(Wu=s["Wu"][:5]), dict(Wd=s["Wd"][:, :7]), dict(x=s["x"].t()), dict(Wu=s["Wu"][:1].expand(24, 16)), dict(x=s["x"].cpu()),
                   dict(activation="tanh"), dict(x=s["x"].double())):
        with pytest.raises(GadError):
            pkg.gated_feed_forward(**{**s, **change})
        if "activation" not in change:
            with pytest.raises(GadError):
                pkg.gated_feed_forward_backward(dy, **{**s, **change}, **saved)
    for change in (dict(h=r.h[:5]), dict(act=r.act.half()), dict(slope=r.slope[:1].expand(6, 24)), dict(grads="q")):
        with pytest.raises(GadError):
            pkg.gated_feed_forward_backward(dy, **s, **{**saved, **change})
    with pytest.raises(GadError):
        pkg.gated_feed_forward_backward(dy[:5], **s, **saved)


def test_refusals_of_the_library():
    """On the host, before anything is enqueued."""
    L = ff._load()
    n = ctypes.c_size_t(0)

    def fwd(**k):
        a = ff._ForwardArgs(dtype=2, cols=16, inner=24, activation=0, rows=5, ldx=16, ldwg=16, ldwu=16, ldwd=24, ldy=16)
        for f, v in k.items():
            setattr(a, f, v)
        return L.gad_gated_feed_forward_workspace_bytes(ctypes.byref(a), ctypes.byref(n))

    def bwd(**k):
        a = ff._BackwardArgs(dtype=2, cols=16, inner=24, rows=5, lddy=16, ldx=16, ldwg=16, ldwu=16, ldwd=24, ldact=24, ldslope=24, ldh=24, dx=256, lddx=16)
        for f, v in k.items():
            setattr(a, f, v)
        return L.gad_gated_feed_forward_backward_workspace_bytes(ctypes.byref(a), ctypes.byref(n))
    assert fwd() == 0 and n.value > 0 and bwd() == 0 and n.value > 0
    assert fwd(rows=0) == 0 and n.value == 0 and bwd(rows=0) == 0 and n.value == 0
    for k in (dict(dtype=3), dict(dtype=-1), dict(cols=0), dict(inner=0), dict(rows=-1), dict(ldx=15), dict(ldwg=15), dict(ldwu=0), dict(ldwd=23), dict(activation=4), dict(ldy=8),
              dict(act=256), dict(act=256, slope=256, h=256, ldact=24, ldslope=24, ldh=23), dict(act=256, slope=256, h=258, ldact=24, ldslope=24, ldh=24)):
        assert fwd(**k) == -1, k
    for k in (dict(dtype=3), dict(cols=0), dict(rows=-1), dict(lddy=15), dict(ldwu=0), dict(ldact=23), dict(ldh=0), dict(lddx=15), dict(dw_down=256, lddwd=23)):
        assert bwd(**k) == -1, k
    for k in (dict(rows=2 ** 31), dict(cols=2 ** 21, ldx=2 ** 21, ldwg=2 ** 21, ldwu=2 ** 21, ldy=2 ** 21), dict(inner=2 ** 21, ldwd=2 ** 21)):
        assert fwd(**k) == -2, k
    assert L.gad_gated_feed_forward_workspace_bytes(None, ctypes.byref(n)) == -1
    # pointers that are missing, and workspaces that are too small or start on no 256 bytes
    a = ff._ForwardArgs(dtype=2, cols=16, inner=24, activation=0, rows=5, ldx=16, ldwg=16, ldwu=16, ldwd=24, ldy=16)
    assert L.gad_gated_feed_forward(ctypes.byref(a), 256, 1 << 30, None) == -1
    a.status = 256
    assert L.gad_gated_feed_forward(ctypes.byref(a), 256, 1 << 30, None) == -1
    a.x = a.w_gate = a.w_up = a.w_down = a.y = 256
    assert L.gad_gated_feed_forward(ctypes.byref(a), 256, 16, None) == -5
    assert L.gad_gated_feed_forward(ctypes.byref(a), 264, 1 << 30, None) == -5
    assert L.gad_gated_feed_forward(ctypes.byref(a), None, 1 << 30, None) == -5
    with pytest.raises(GadError):
        import torch
        pkg.gated_feed_forward(torch.ones(2, 2), torch.ones(2, 2), torch.ones(2, 2), torch.ones(2, 2))


def test_kernels_wait_for_the_one_in_front():
    """Every kernel of a call may come up before the one in front of it has ended."""
    import os
    import re
    from test_launch_contract import kernels, CSRC
    text = re.sub(r"//[^\n]*", "", "".join(open(os.path.join(CSRC, f)).read() for f in ("gated_few.cuh", "gated_gemm.cuh", "gated_launch.cuh", "gated_skinny.cuh", "gated.cu")))
    bodies = kernels(text)
    chained = set(bodies) - {"gated_zero_kernel", "gated_empty_kernel"}
    assert {"gated_gemm_kernel", "gated_join_kernel", "gated_hidden_join_kernel", "gated_pack_kernel", "skinny_kernel", "skinny_join_kernel", "few_rows_kernel"} <= chained
    for name in chained:
        assert "pdl_wait();" in bodies[name], name
