"""Layer norm and its backward pass against the definition in 64 bits.

Tolerances count roundings, u = 2^-24 a step of fp32 arithmetic and eps/2 the last rounding to the output's type.  A sum here is a chain of at most
16 vectors x 8 values in a thread, 5 shuffles and 32 warps (rows of more than 8192 or 32 768 values: cols / 1024 instead of the 128), so its error is at most
CHAIN u times the sum of magnitudes; a product or difference more adds a step."""
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import GadError

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def chain(cols):
    return 170 + cols // 1024


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def tiny_step(dtype):
    """Half a step of the type's subnormals."""
    import torch
    return {torch.float16: 2.0 ** -25}.get(dtype, 2.0 ** -134)


def make(rows, cols, dtype, seed, pad=0, offset=0, shift=0.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    m = torch.randn(rows, cols, generator=g, dtype=torch.float64) * (0.2 + torch.rand(rows, 1, generator=g, dtype=torch.float64)) + shift
    buf = torch.zeros(rows * (cols + pad) + offset, dtype=dtype, device="cuda")
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(m)
    return v


def check(got, want, bound, what):
    import torch
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), "%s: over its bound by %.3g" % (what, off.max().item())
    assert torch.isfinite(got.float()).all()


# rows, cols, pad of the row stride, elements the first row starts behind its allocation
SHAPES = [(1, 1, 0, 0), (3, 2, 0, 0), (5, 31, 0, 0), (7, 64, 0, 0), (2708, 256, 0, 0), (4, 129, 7, 0), (9, 500, 12, 0), (33, 1000, 0, 1), (6, 1024, 8, 0),
          (5, 1433, 0, 0), (3, 2048, 0, 0), (700, 2052, 4, 0), (2, 4096, 0, 0), (2, 8192, 0, 0), (3, 8191, 1, 0), (3, 8200, 0, 1), (2, 16384, 0, 0), (2, 32768, 0, 0), (2, 40000, 0, 0)]


@gpu
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,cols,pad,offset", SHAPES)
@pytest.mark.parametrize("p32", [True, False])
def test_forward_and_backward(rows, cols, pad, offset, dtype, p32):
    import torch
    dt = getattr(torch, dtype)
    pt = torch.float32 if p32 else dt
    x, dy = make(rows, cols, dt, 1, pad, offset, shift=3.0), make(rows, cols, dt, 2, pad, offset)
    g = torch.Generator().manual_seed(3)
    gamma = (1 + 0.3 * torch.randn(cols, generator=g)).to(pt).cuda()
    beta = torch.randn(cols, generator=g).to(pt).cuda()
    y, mean, rstd = pkg.layer_norm(x, gamma, beta, eps=1e-5)
    X, D, G, B = x.double(), dy.double(), gamma.double(), beta.double()
    mu = X.mean(1, keepdim=True)
    var = (X - mu).square().mean(1, keepdim=True)
    rs = 1 / (var + 1e-5).sqrt()
    n = chain(cols)
    amax = X.abs().amax(1, keepdim=True)
    dmu = (n + 2) * U * amax
    # relative error of the deviation: half that of the variance, a sum of squares of differences with an error of dmu + u |x| each
    drs = (n + 8) * U + (dmu + U * amax).square() * rs.square() + 2 * (dmu + U * amax) * U * n * rs
    check(mean, mu[:, 0], dmu[:, 0] + 1e-45, "mean")
    check(rstd, rs[:, 0], (drs * rs)[:, 0], "rstd")
    h = (X - mu) * rs
    want = h * G + B
    bound = ((dmu + U * amax) * rs + h.abs() * (drs + 2 * U)) * G.abs() + 2 * U * (want.abs() + B.abs())
    check(y, want, bound + half_step(dt) * (want.abs() + bound) + tiny_step(dt), "y")

    dx, dgamma, dbeta = pkg.layer_norm_backward(dy, x, mean, rstd, gamma)
    # from here the statistics are inputs
    mu, rs = mean.double()[:, None], rstd.double()[:, None]
    h, g2 = (X - mu) * rs, D * G
    want = rs * (g2 - g2.mean(1, keepdim=True) - h * (g2 * h).mean(1, keepdim=True))
    size = rs * (g2.abs() + g2.abs().mean(1, keepdim=True) + h.abs() * (g2 * h).abs().mean(1, keepdim=True))
    bound = (n + 12) * U * size
    check(dx, want, bound + half_step(dt) * (want.abs() + bound) + tiny_step(dt), "dx")
    steps = (rows // 512 + 110) * U
    for got, terms, what in ((dgamma, D * h, "dgamma"), (dbeta, D, "dbeta")):
        want, bound = terms.sum(0), (steps + 3 * U) * terms.abs().sum(0)
        check(got, want, bound + half_step(pt) * (want.abs() + bound) + tiny_step(pt), what)
    assert dx.dtype == dt and dgamma.dtype == dbeta.dtype == pt and y.dtype == dt


@gpu
@pytest.mark.parametrize("cols", [16, 300, 2000])
def test_gradients_are_differences_of_the_definition(cols):
    import torch
    rows = 6
    x, dy = make(rows, cols, torch.float32, 5, shift=0.5), make(rows, cols, torch.float32, 6)
    g = torch.Generator().manual_seed(7)
    gamma, beta = torch.randn(cols, generator=g).cuda(), torch.randn(cols, generator=g).cuda()

    def value(X, G, B):
        mu = X.mean(1, keepdim=True)
        return (dy.double() * ((X - mu) / ((X - mu).square().mean(1, keepdim=True) + 1e-5).sqrt() * G + B)).sum()

    y, mean, rstd = pkg.layer_norm(x, gamma, beta)
    dx, dgamma, dbeta = pkg.layer_norm_backward(dy, x, mean, rstd, gamma)
    at = [x.double(), gamma.double(), beta.double()]
    for i, grad in enumerate((dx, dgamma, dbeta)):
        for seed in range(3):
            v = torch.randn(at[i].shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).cuda()
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-4 * v, at[i] - 1e-4 * v
            diff = (value(*up) - value(*down)) / 2e-4
            # third derivatives of order 1 times 1e-8, cancellation 1e-16 / 1e-4, and the fp32 gradients: chain(cols) u
            tol = (1e-7 + chain(cols) * U) * (grad.double().norm() * v.norm() + dy.double().norm())
            assert abs(diff - (grad.double() * v).sum()) <= tol


@gpu
def test_rows_of_a_single_value_large_means_and_no_parameters():
    import torch
    x = torch.full((4, 700), 7.0, device="cuda")
    y, mean, rstd = pkg.layer_norm(x)
    assert torch.equal(y, torch.zeros_like(x)) and torch.equal(mean, x[:, 0]) and torch.allclose(rstd, torch.full((4,), 1e-5 ** -0.5, device="cuda"), rtol=1e-6, atol=0)
    dx, dgamma, dbeta = pkg.layer_norm_backward(torch.ones_like(x), x, mean, rstd)
    assert torch.equal(dgamma, torch.zeros(700, device="cuda")) and torch.equal(dbeta, torch.full((700,), 4.0, device="cuda"))
    assert dx.abs().max() <= 1024 * U * rstd[0]
    # a mean 10^4 times the deviation: what is left is the rounding of x itself and of the mean
    x = (1e4 + torch.randn(8, 4096, dtype=torch.float64)).float().cuda()
    y, mean, rstd = pkg.layer_norm(x)
    X = x.double()
    want = (X - X.mean(1, keepdim=True)) / (X.var(1, correction=0, keepdim=True) + 1e-5).sqrt()
    assert (y.double() - want).abs().max() <= (chain(4096) + 2) * U * 1.0001e4 * 1.1


@gpu
def test_a_row_with_nan_or_infinity_stays_alone():
    import torch
    x = make(6, 512, torch.bfloat16, 1)
    clean, _, _ = pkg.layer_norm(x)
    x[2, 100], x[4, 5] = math.nan, math.inf
    y, mean, rstd = pkg.layer_norm(x)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
    dx, _, _ = pkg.layer_norm_backward(torch.ones_like(x), x, mean, rstd)
    assert torch.isfinite(dx[keep].float()).all() and torch.isnan(dx[2].float()).all()


@gpu
def test_no_rows_broadcast_gradients_streams_and_equal_bits():
    import torch
    e = torch.empty(0, 64, device="cuda")
    y, mean, rstd = pkg.layer_norm(e)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dgamma, dbeta = pkg.layer_norm_backward(e, e, mean, rstd)
    assert dx.shape == (0, 64) and not dgamma.any() and not dbeta.any()
    x = make(1000, 384, torch.float16, 1)
    gamma = torch.rand(384, device="cuda").half()
    y, mean, rstd = pkg.layer_norm(x, gamma)
    one = torch.ones(1, 384, device="cuda", dtype=torch.float16)
    a = pkg.layer_norm_backward(one.expand(1000, 384), x, mean, rstd, gamma)            # a broadcast upstream gradient
    b = pkg.layer_norm_backward(one.expand(1000, 384).contiguous(), x, mean, rstd, gamma)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = pkg.layer_norm_backward(one.expand(1000, 384), x, mean, rstd, gamma, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(u, v) for u, v in zip(a, c))
    only, dg, db = pkg.layer_norm_backward(one.expand(1000, 384), x, mean, rstd, gamma, param_grads=False)
    assert torch.equal(only, a[0]) and dg is None and db is None


@gpu
def test_captured_and_replayed():
    import torch
    x, dy = make(300, 1024, torch.bfloat16, 1), make(300, 1024, torch.bfloat16, 2)
    gamma, beta = torch.rand(1024, device="cuda"), torch.rand(1024, device="cuda")

    def step():
        y, mean, rstd = pkg.layer_norm(x, gamma, beta)
        return (y, mean, rstd) + pkg.layer_norm_backward(dy, x, mean, rstd, gamma)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for seed in (5, 6):
        x.copy_(make(300, 1024, torch.bfloat16, seed))
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        assert all(torch.equal(u, v) for u, v in zip(kept, step()))


def test_refusals_on_the_host():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(GadError):
        pkg.layer_norm(x)                                       # not on a GPU
    with pytest.raises(GadError):
        pkg.layer_norm_backward(x, x, torch.zeros(4), torch.zeros(4))
    L = pkg.load()
    n = __import__("ctypes").c_size_t(0)
    import ctypes
    assert L.gad_layer_norm_backward_workspace_bytes(ctypes.c_int64(10), ctypes.c_int32(16), ctypes.byref(n)) == 0 and n.value == 10 * 2 * 16 * 4
    assert L.gad_layer_norm_backward_workspace_bytes(ctypes.c_int64(-1), ctypes.c_int32(16), ctypes.byref(n)) == -1
    one = ctypes.c_void_p(256)
    i64, i32, f = ctypes.c_int64, ctypes.c_int32, ctypes.c_float

    def forward(ldx=8, rows=4, cols=8, dtype=0, p=0, eps=1e-5, ldy=8, x=one):
        return L.gad_layer_norm(x, i64(ldx), i64(rows), i32(cols), i32(dtype), None, None, i32(p), f(eps), one, i64(ldy), one, one, None)

    assert forward(rows=0) == 0
    for bad in (dict(cols=0), dict(rows=-1), dict(rows=1 << 31), dict(dtype=3), dict(dtype=1, p=2), dict(eps=-1.0), dict(eps=math.nan), dict(ldx=7), dict(ldy=7), dict(ldy=0), dict(x=None)):
        assert forward(**bad) == -1, bad

    def backward(dtype=0, p=0, ld=8, ws=one, nws=1 << 20, dg=one):
        return L.gad_layer_norm_backward(one, i64(ld), one, i64(8), i64(4), i32(8), i32(dtype), None, i32(p), one, one, one, i64(8), dg, None, ws, ctypes.c_size_t(nws), None)

    assert backward(dtype=2, p=1) == -1 and backward(ld=3) == -1 and backward(ws=None) == -5 and backward(nws=255) == -5


@gpu
def test_refusals_of_tensors():
    import torch
    x = torch.zeros(4, 8, device="cuda")
    v = torch.zeros(8, device="cuda")
    r = torch.zeros(4, device="cuda")
    for bad in (dict(x=x.double()), dict(x=x[0]), dict(x=x.t()), dict(x=x, gamma=v[:7]), dict(x=x, gamma=v.half()), dict(x=x, gamma=v, beta=v.double()), dict(x=x.half(), gamma=v, beta=v.half()),
                dict(x=x, gamma=v.cpu()), dict(x=x, eps=-1.0), dict(x=torch.zeros(4, 0, device="cuda")), dict(x=torch.zeros(64, device="cuda").as_strided((4, 8), (4, 1)))):
        with pytest.raises(GadError):
            pkg.layer_norm(**bad)
    for bad in ((x.half(), x, r, r), (x[:3], x, r, r), (x, x, r[:3], r), (x, x, r, r.double()), (x, x, None, r), (x, x, r, r, v.half())):
        with pytest.raises(GadError):
            pkg.layer_norm_backward(*bad)
