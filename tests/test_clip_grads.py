"""Global norm and clipping of gradients against the formulas in 64 bits.

Tolerances: the norm's squares are summed in fp32 over at most 32 values of a thread (33 roundings of 2^-24, halved by the square root) and in fp64 above, and rounded to fp32 once: 18 x 2^-24.
The factor carries that and one rounding, the product one more, the result's type half a step."""
import ctypes
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import GadError
from paper_2110_02987_b200 import grads as gr

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def norm_of(grads):
    return math.sqrt(sum(float((t.double() * t.double()).sum()) for t in grads))


def held(got, want):
    import torch
    f = torch.finfo(got.dtype)
    tol = 20 * U * want.abs() + f.eps / 2 * want.abs().clamp(min=f.tiny) * (1 + 20 * U)
    assert got.shape == want.shape and bool(((got.double() - want).abs() <= tol).all())


def make(shapes, dtype, seed=0, scale=0.1, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    kinds = ["float32", "float16", "bfloat16"]
    out = []
    for i, (r, c) in enumerate(shapes):
        dt = getattr(torch, dtype if dtype != "mixed" else kinds[i % 3])
        m = torch.full((r, c + pad), math.nan, dtype=dt, device="cuda")[:, :c]
        m.copy_(torch.randn(r, c, generator=g) * scale)
        out.append(m)
    return out


SHAPES = {"one": [(1, 1)], "few": [(3, 5), (1, 17), (64, 64), (0, 4), (1, 8192)], "odd": [(33, 1433), (1, 8193), (257, 31), (8193, 1), (2, 20000), (5, 8192)], "many": [(7, i + 1) for i in range(100)],
          "more": [(3, i % 19 + 1) for i in range(1000)], "large": [(2000, 2047), (1, 5_000_001), (513, 4096)]}


@gpu
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16", "mixed"])
@pytest.mark.parametrize("shapes", list(SHAPES))
def test_norm_and_clipping(shapes, dtype, pad):
    import torch
    grads = make(SHAPES[shapes], dtype, len(shapes), pad=pad)
    n = norm_of(grads)
    assert abs(pkg.grad_norm(grads).item() - n) <= 18 * U * n
    for factor in (0.3, 1.5):
        f = min(1.0, factor)
        want = [t.double() * f for t in grads]
        # into tensors of the same type and of fp32, then in place
        for out in ([torch.full_like(t, 7) for t in grads], [torch.full(t.shape, 7.0, device="cuda") for t in grads]):
            before = [t.clone() for t in grads]
            got = pkg.clip_grads(grads, n * factor, out=out)
            assert abs(got.item() - n) <= 18 * U * n and all(torch.equal(a, b) for a, b in zip(before, grads))
            for t, w in zip(out, want):
                held(t, w)
                assert factor < 1 or torch.equal(t, w.to(t.dtype))
        mine = [t.clone(memory_format=torch.preserve_format) if not pad else make([t.shape], str(t.dtype)[6:], 0, pad=pad)[0].copy_(t) for t in grads]
        wide = [t._base for t in mine]
        got = pkg.clip_grads(mine, n * factor)
        assert abs(got.item() - n) <= 18 * U * n
        for t, w in zip(mine, want):
            held(t, w)
        if pad:                                                                # what lies between the rows is left as it was
            for b, t in zip(wide, mine):
                assert bool(b[:, t.shape[1]:].isnan().all())


@gpu
def test_long_chunks():
    """Enough values for chunks of 32 768: odd sizes, rows of a wider matrix, in place."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    grads = [torch.randn(90_000_001, generator=g, device="cuda").bfloat16(), torch.randn(7000, 10_009, generator=g, device="cuda").half()[:, :9999], torch.randn(33_333, generator=g, device="cuda")]
    n = norm_of(grads)
    want = [t.double() * 0.25 for t in grads]
    rest = grads[1]._base[:, 9999:].clone()
    assert abs(pkg.clip_grads(grads, n / 4).item() - n) <= 36 * U * n          # (128 values a thread in two sums: 65 roundings, halved)
    for t, w in zip(grads, want):
        held(t, w)
    assert torch.equal(grads[1]._base[:, 9999:], rest)


@gpu
def test_layouts():
    """Transposed matrices, columns of one matrix, tensors of more dimensions, starts off 16 bytes, a matrix with rows into a dense one."""
    import torch
    base = torch.randn(200, 300, device="cuda")
    flat = torch.randn(1003, device="cuda")
    grads = [base.t()[:100], base.t()[100:], torch.randn(4, 5, 6, device="cuda"), flat[1:1000], torch.randn((), device="cuda"), torch.randn(50, 7, device="cuda").t(), torch.randn(20, 40, device="cuda")[:, :33]]
    want = [t.double() * 0.5 for t in grads]
    n = norm_of(grads)
    out = [torch.empty_strided(t.shape, t.stride(), device="cuda") if t.dim() == 2 else torch.empty_like(t) for t in grads[:6]] + [torch.empty(20, 33, device="cuda")]
    pkg.clip_grads(grads, n * 0.5, out=out)
    for t, w in zip(out, want):
        held(t, w)
    dense = torch.randn(20, 33, device="cuda")
    wide = torch.empty(20, 40, device="cuda")[:, :33]
    pkg.clip_grads([dense, None], math.inf, out=[wide, None])
    assert torch.equal(dense, wide)
    pkg.clip_grads(grads, n * 0.5)
    for t, w in zip(grads, want):
        held(t, w)
    assert bool(flat[0] != 0) and bool(flat[1000:].abs().max() > 0)


@gpu
@pytest.mark.parametrize("dtype,value", [("float32", 1e30), ("float32", 3e-30), ("float32", 1e-44), ("bfloat16", 1e25), ("bfloat16", 1e-30), ("float16", 6e-8), ("float16", 60000.0)])
def test_squares_neither_overflow_nor_vanish(dtype, value):
    import torch
    grads = [torch.full((1000,), value, device="cuda").to(getattr(torch, dtype)), torch.zeros(70000, device="cuda"), torch.full((3, 5), value, device="cuda").to(getattr(torch, dtype))[:, 1:]]
    n = norm_of(grads)
    assert n > 0
    got = pkg.clip_grads(grads, n / 2, out=[torch.empty(t.shape, device="cuda") for t in grads])
    assert abs(got.item() - n) <= 18 * U * n + 2.0 ** -149


@gpu
def test_norms_that_are_zero_or_not_finite():
    import torch
    z = [torch.zeros(100, device="cuda"), torch.zeros(5, 5, device="cuda", dtype=torch.bfloat16)]
    assert pkg.clip_grads(z, 1.0).item() == 0 and pkg.clip_grads(z, 0.0).item() == 0 and not z[0].any()
    for bad in (math.inf, -math.inf, math.nan):
        g = [torch.ones(1000, device="cuda"), torch.full((20000,), 2.0, device="cuda", dtype=torch.float16)]
        g[1][7] = bad
        keep = [t.clone() for t in g]
        out = [torch.zeros_like(t) for t in g]
        n = pkg.clip_grads(g, 1.0, out=out)
        assert not math.isfinite(n.item()) and math.isnan(n.item()) == math.isnan(bad)
        assert all(torch.equal(a.view(torch.int32 if a.element_size() == 4 else torch.int16), b.view(torch.int32 if a.element_size() == 4 else torch.int16)) for a, b in zip(out, keep))
    g = [torch.ones(1000, device="cuda")]
    pkg.clip_grads(g, 0.0)
    assert not g[0].any()


@gpu
def test_equal_calls_streams_and_graphs():
    import torch
    grads = make(SHAPES["odd"] + SHAPES["few"], "mixed", 3)
    out = [torch.empty_like(t) for t in grads]
    n = pkg.clip_grads(grads, 0.5, out=out)
    again = [torch.empty_like(t) for t in grads]
    assert torch.equal(n, pkg.clip_grads(grads, 0.5, out=again)) and all(torch.equal(a, b) for a, b in zip(out, again))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(t) for t in grads] for _ in range(6)]
    norms = [pkg.clip_grads(grads, 0.5, out=o, stream=streams[i % 2]) for i, o in enumerate(outs)]
    torch.cuda.synchronize()
    assert all(torch.equal(m, n) for m in norms) and all(torch.equal(a, b) for o in outs for a, b in zip(o, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m = pkg.clip_grads(grads, 0.5, out=again)
    grads[0].mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(m, pkg.clip_grads(grads, 0.5, out=out)) and not torch.equal(m, n) and all(torch.equal(a, b) for a, b in zip(out, again))


@gpu
def test_refusals_of_tensors():
    import torch
    a, b = torch.ones(10, 10, device="cuda"), torch.ones(10, 10, device="cuda")
    for bad in ([], [None], [torch.ones(3)], [a, torch.ones(3)], [a.double()], [a, a], [a, a[2:4]], [a, a.t()], [a[:, :5], a[:, 4:]], [a[::2, ::2]], [a[:1].expand(3, 10)], a, [a.int()]):
        with pytest.raises(GadError):
            pkg.clip_grads(bad, 1.0)
    for out in ([b], [b, a], [b, b], [b[:5], b], [b.half(), b], [b.t()[:, :], torch.ones(10, 10, device="cuda")[:, :]][:1] + [a]):
        with pytest.raises(GadError):
            pkg.clip_grads([a, torch.ones(10, 10, device="cuda")], 1.0, out=out)
    for m in (-1.0, math.nan):
        with pytest.raises(GadError):
            pkg.clip_grads([a], m)
    assert pkg.grad_norm([a, a]).item() == pytest.approx(math.sqrt(200))
    pkg.clip_grads([a[:, :5], a[:, 5:]], 1.0)


def test_refusals_of_the_library():
    """On the host, before anything is enqueued."""
    L = gr._load()
    n = ctypes.c_size_t(0)
    assert L.gad_clip_grads_workspace_bytes(5, ctypes.byref(n)) == 0 and n.value > 0
    assert L.gad_clip_grads_workspace_bytes(-1, ctypes.byref(n)) == -1 and L.gad_clip_grads_workspace_bytes(2 ** 21, ctypes.byref(n)) == -2

    def call(*entries, max_norm=1.0, norm=256, ws=256, size=1 << 30):
        return L.gad_clip_grads(gr._packer(len(entries)).pack(*[v for e in entries for v in e]), len(entries), max_norm, norm, ws, size, None)
    good = (4096, 0, 0, 2, 8, 8, 4096, 8)
    assert call(good, ws=None) == -5 and call(good, size=16) == -5 and call(good, ws=264) == -5
    for e in ((4096, 3, 3, 2, 8, 8, 4096, 8), (4096, 0, 0, -1, 8, 8, 4096, 8), (0, 0, 0, 2, 8, 8, 4096, 8), (4098, 0, 0, 2, 8, 8, 4098, 8), (4096, 0, 0, 2, 8, 7, 4096, 8), (4096, 0, 1, 2, 8, 8, 8192, 8),
              (4096, 0, 0, 2, 8, 8, 4096, 9), (4096, 1, 0, 2, 8, 8, 4096, 8), (4096, 0, 0, 2, 8, 8, 4128, 8), (4096, 0, 0, 2, 8, 8, 8194, 8)):
        assert call(e) == -1, e
    assert call((4096, 0, 0, 2 ** 21, 2 ** 21, 2 ** 21, 4096, 2 ** 21)) == -2
    assert call(good, good) == -1 and call(good, norm=None) == -1 and call(good, max_norm=-1.0) == -1 and call(good, max_norm=math.nan) == -1
    # columns of one matrix are tensors of their own; where they meet they are refused
    assert call((4096, 0, 0, 4, 8, 32, 4096, 32), (4096 + 32, 0, 0, 4, 24, 32, 4096 + 32, 32), ws=None) == -5
    assert call((4096, 0, 0, 4, 9, 32, 4096, 32), (4096 + 32, 0, 0, 4, 24, 32, 4096 + 32, 32), ws=None) == -1
    assert call((4096, 0, 0, 4, 8, 32, 4096, 32), (4096 + 32, 0, 0, 4, 25, 32, 4096 + 32, 32), ws=None) == -1


def test_kernels_wait_for_the_one_in_front():
    import os
    import re
    from test_launch_contract import kernels, CSRC
    bodies = kernels(re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "grad_clip.cu")).read()))
    assert set(bodies) == {"grad_squares_kernel", "grad_scale_kernel"}
    for name, body in bodies.items():
        assert "pdl_wait();" in body, name
