"""Clipped policy loss with a KL term against its definition in 64 bits, with its gradients.

Tolerances as for the loss over many classes: u = 2^-24; a logit is off by ``steps(K)`` 2u times the sum of its terms' magnitudes, at most d; a log-probability by 2 d and 4 u of the largest |z| (its sum, logarithm and
the scaling by log2 e); r = exp(lp - old) by that relatively and 4 u more; losses follow by their slopes.  A probability is off relatively by 2 d + e_lp + 16 u, with 16-bit operands by 2^-12 ln 2 more (its code); G
is rounded to the operand type, the result once more, and the sums of its products are off by ``steps`` 2u of their magnitudes.  No ratio is drawn nearer to a border than its own tolerance could carry it across."""
import ctypes
import math
import types

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import GadError
from paper_2110_02987_b200 import head

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def steps(K, dtype):
    import torch
    return 2 * U * (K / 16 + K / 256 + 16 if dtype == torch.float32 else K / 16 + 8)


def half(v, dtype):
    import torch
    f = torch.finfo(dtype)
    return f.eps / 2 * v.abs().clamp(min=f.tiny)


def matrix(rows, cols, dtype, g, scale=1.0, pad=0):
    import torch
    m = torch.randn(rows, cols, generator=g, dtype=torch.float64) * scale
    v = torch.full((rows, cols + pad), math.nan, dtype=dtype, device="cuda")[:, :cols]
    v.copy_(m)
    return v


def make(N, D, V, dtype, seed=0, bias=False, weights=False, ignored=0.0, ref=True, pad=0, int64=False, low=0.2, high=0.28):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)
    s = dict(H=matrix(N, D, dt, g, 1.0, pad), W=matrix(V, D, dt, g, 1.5 / math.sqrt(D), pad))
    actions = torch.randint(0, V, (N,), generator=g)
    b = torch.randn(V, generator=g).to(dt).cuda() if bias else None
    z = s["H"].double() @ s["W"].double().t() + (b.double() if bias else 0)
    lp = z.log_softmax(1).gather(1, actions.cuda()[:, None])[:, 0].cpu()
    moved = 0.3 * torch.randn(N, generator=g, dtype=torch.float64)
    for border in (math.log(1 - low), math.log(1 + high)):
        off = moved - border
        moved = torch.where(off.abs() < 2e-3, border + 2e-3 * torch.where(off < 0, -1.0, 1.0), moved)
    drop = torch.rand(N, generator=g) < ignored
    old, adv = (lp - moved).float(), torch.randn(N, generator=g)
    nan = torch.where(drop, math.nan, 0.0)                                     # what rows that do not count hold is no number
    return dict(s, actions=torch.where(drop, -7, actions).to(torch.int64 if int64 else torch.int32).cuda(), old_logp=(old + nan).cuda(), advantages=(adv + nan).cuda(),
                ref_logp=((lp + 0.4 * torch.randn(N, generator=g)).float() + nan).cuda() if ref else None, clip=(low, high), kl_weight=0.1 if ref else 0.0, bias=b,
                row_weights=(torch.rand(N, generator=g) * 3 - 1).cuda() if weights else None)


def reference(H, W, actions, old_logp, advantages, ref_logp=None, clip=(0.2, 0.2), kl_weight=0.0, bias=None, row_weights=None, mean=True, scale=1.0):
    """Values and tolerances of every output."""
    import torch
    dt = H.dtype
    low, high = clip
    h, w = H.double(), W.double()
    N, D = h.shape
    V = w.shape[0]
    has = actions >= 0
    h = torch.where(has[:, None], h, 0.0)
    z = h @ w.t() + (bias.double() if bias is not None else 0)
    d = steps(D, dt) * (h.abs() @ w.abs().t()).max(1).values + 4 * U * z.abs().max(1).values
    at = actions.clamp(min=0).long()[:, None]
    lp = z.log_softmax(1).gather(1, at)[:, 0]
    e_lp = 2 * d + 4 * U * (lp.abs() + 1)
    take = lambda t: torch.where(has, t.double(), 0.0)  # noqa: E731
    A, old = take(advantages), take(old_logp)
    r = torch.exp(lp - old)
    e_r = r * (torch.expm1(e_lp + 4 * U * (1 + (lp - old).abs())))
    plain, held = r * A, r.clamp(1 - low, 1 + high) * A
    clipped = plain > held
    l = torch.where(clipped, -held, -plain)
    slope = torch.where(clipped, 0.0, -plain)
    e_l = A.abs() * e_r + 4 * U * l.abs()
    e_s = torch.where(clipped, 0.0, e_l)
    if ref_logp is not None:
        x = take(ref_logp) - lp
        l = l + kl_weight * (torch.expm1(x) - x)
        slope = slope - kl_weight * torch.expm1(x)
        e_x = e_lp + U * (x.abs() + 1)
        e_l = e_l + kl_weight * (torch.exp(x) + 1) * (2 * e_x) + 4 * U * (l.abs() + kl_weight * (x.abs() + 1))
        e_s = e_s + kl_weight * torch.exp(x) * 2 * e_x + 4 * U * slope.abs()
    l, slope, e_l, e_s, lp, e_lp = (torch.where(has, t, 0.0) for t in (l, slope, e_l, e_s, lp, e_lp))
    f = torch.ones(N, dtype=torch.float64, device="cuda") if row_weights is None else row_weights.double()
    f = torch.where(has, f, 0.0) * scale / (max(1, int(has.sum())) if mean else 1)
    loss, e_loss = (f * l).sum().reshape(1), (f.abs() * e_l).sum().reshape(1) + 4 * U * (f * l).abs().sum()
    p = z.softmax(1)
    c = f * slope
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    G = c[:, None] * (one - p)
    rel = (d + e_lp + 16 * U)[:, None] + (0 if dt == torch.float32 else 2.0 ** -12 * math.log(2))
    size = c.abs()[:, None] * (one + p)
    e_G = (f.abs() * e_s + 4 * U * c.abs())[:, None] * (one + p) + c.abs()[:, None] * p * rel + 4 * U * size
    eb = e_G.sum(0) + 2 * U * (N / 32 + 16) * size.sum(0)
    if dt == torch.float16:      # in units of the largest coefficient: fp16's smallest step of it is 2^-24 / 2^14
        e_G = e_G + 2.0 ** -39 * c.abs().max()
    e_G = e_G + (torch.finfo(dt).eps / 2 if dt != torch.float32 else 2.0 ** -23) * (G.abs() + e_G)
    out = types.SimpleNamespace(loss=(loss, e_loss), row_loss=(l, e_l), logp=(lp, e_lp))
    for name, m, e, v in (("dH", G, e_G, w), ("dW", G.t(), e_G.t(), h)):
        want = m @ v
        setattr(out, name, (want, e @ v.abs() + steps(m.shape[1], dt) * ((m.abs() + e) @ v.abs()) + half(want, dt) * (1 + 2.0 ** -8)))
    out.db = (G.sum(0), eb + half(G.sum(0), dt) * (1 + 2.0 ** -8))
    return out


def near(got, want, names=("loss", "row_loss", "logp", "dH", "dW", "db")):
    for name in names:
        t = getattr(got, name)
        if t is None:
            continue
        v, tol = getattr(want, name)
        assert t.shape == v.shape, name
        off = (t.double() - v).abs() - tol
        assert bool((off <= 1e-30).all()), "%s: %g over its tolerance of %g" % (name, float(off.max()), float(tol.max()))


SIZES = [(1, 1, 2), (1, 64, 1000), (3, 33, 7), (5, 200, 129), (16, 128, 300), (17, 57, 1001), (40, 500, 64), (200, 64, 5000), (300, 136, 777), (513, 256, 1024)]


@gpu
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_loss_and_gradients(N, D, V, dtype):
    i = SIZES.index((N, D, V))
    s = make(N, D, V, dtype, i, bias=i % 2 == 0, weights=i % 3 == 1, ignored=0.3 if N > 2 else 0.0, ref=i % 4 != 1, pad=(0, 5, 8)[i % 3], int64=i % 2 == 1)
    want = reference(**s)
    near(pkg.policy_loss(**s).check(), want)
    no = pkg.policy_loss(**s, grads=False).check()
    assert no.dH is None and no.dW is None and no.db is None
    near(no, want, ("loss", "row_loss", "logp"))
    for grads in ("H", "W"):
        near(pkg.policy_loss(**s, grads=grads).check(), want)
    near(pkg.policy_loss(**s, mean=False, scale=0.5).check(), reference(**s, mean=False, scale=0.5))


@gpu
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,D,V", [(300, 1100, 700), (130, 2100, 1000), (65, 4096, 300), (520, 1030, 257)])
def test_long_rows(N, D, V, dtype):
    """Logits that are added up in chunks, in tiles of 256 columns, the last of them ragged."""
    s = make(N, D, V, dtype, N, bias=N % 4 == 0, weights=N == 130, ignored=0.2, pad=8 if N == 65 else 0)
    want = reference(**s)
    near(pkg.policy_loss(**s).check(), want)
    near(pkg.policy_loss(**s, grads=False).check(), want, ("loss", "row_loss", "logp"))


@gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("N,D,V", [(5, 64, 3), (6, 33, 127), (16, 1200, 129), (17, 700, 40_000), (33, 8, 300), (48, 2056, 1001), (64, 520, 20_000), (65, 64, 500)])
def test_scores_of_a_few_rows(N, D, V, dtype):
    """No gradients: log-probabilities and losses of serving, every width of the instruction, long rows in chunks."""
    import torch
    s = make(N, D, V, dtype, N, bias=N % 2 == 0, weights=N % 3 == 0, ignored=0.3, ref=N % 4 != 1)
    want = reference(**s)
    near(pkg.policy_loss(**s, grads=False).check(), want, ("loss", "row_loss", "logp"))
    if s["bias"] is not None and V > 3:                          # classes that are taken out
        s["bias"][1::3] = -math.inf
        s["actions"] = torch.where((s["actions"] % 3 == 1) & (s["actions"] >= 0), s["actions"] - 1, s["actions"])
        z = s["H"].double() @ s["W"].double().t() + s["bias"].double()
        lp = z.log_softmax(1).gather(1, s["actions"].clamp(min=0).long()[:, None])[:, 0]
        got = pkg.policy_loss(**s, grads=False).logp
        assert float((got.double() - torch.where(s["actions"] >= 0, lp, 0.0)).abs().max()) <= float(want.logp[1].max()) * 2
    bad = s["H"].clone()
    if bool((s["actions"] >= 0).any()):
        row = int((s["actions"] >= 0).nonzero()[0, 0])
        bad[row, D // 2] = math.nan
        r = pkg.policy_loss(**dict(s, H=bad), grads=False)
        assert bool(r.logp[row].isnan()) and int(r.logp.isnan().sum()) == 1


@gpu
def test_a_clipped_row_has_no_gradient_but_that_of_the_divergence():
    import torch
    s = make(64, 48, 100, "float32", 3, ref=False)
    lp = -pkg.class_loss(s["H"], s["W"], s["actions"], grads=False).row_loss
    s["advantages"] = torch.where(torch.arange(64, device="cuda") % 2 == 0, 1.0, -1.0)
    s["old_logp"] = lp - s["advantages"]                        # r is e where A > 0 and 1 / e where A < 0: all clipped
    r = pkg.policy_loss(**s).check()
    assert not r.dH.any() and not r.dW.any()
    assert torch.equal(r.row_loss, torch.where(s["advantages"] > 0, -torch.tensor(1.28, device="cuda"), 1 - torch.tensor(0.2, device="cuda")))
    s["old_logp"] = lp + s["advantages"]                        # the other way: none is clipped
    near(pkg.policy_loss(**s).check(), reference(**s))
    s["clip"] = (1.0, math.inf)                                 # no borders at all
    near(pkg.policy_loss(**s).check(), reference(**s))
    s.update(clip=0.0, ref_logp=lp + 0.5, kl_weight=1.0, old_logp=lp - s["advantages"])
    s["clip"] = (0.0, 0.0)
    near(pkg.policy_loss(**s).check(), reference(**s))


@gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_coefficients_of_any_size(dtype):
    """Ratios far from one where nothing holds them (A < 0, r large), and a divergence that explodes: the gradients' scale follows the largest coefficient."""
    import torch
    s = make(300, 64, 200, dtype, 5, ref=False)
    s["advantages"] = -s["advantages"].abs() - 0.1
    s["old_logp"] = s["old_logp"] - 9                           # r up to e^9 and more
    near(pkg.policy_loss(**s).check(), reference(**s))
    s = make(300, 64, 200, dtype, 6)
    s["ref_logp"] = s["ref_logp"] + 8
    near(pkg.policy_loss(**s).check(), reference(**s))
    s = make(300, 64, 200, dtype, 7)
    s["advantages"] = s["advantages"] * 1e-6                    # and small ones
    s["kl_weight"] = 1e-7
    near(pkg.policy_loss(**s).check(), reference(**s))


@gpu
def test_blocks_of_rows_have_scales_of_their_own(monkeypatch):
    """More logits than are held at once: blocks of rows, the coefficients of the second a thousand times those of the first."""
    import torch
    N, D, V = 6000, 64, 200_000
    for dtype in ("float16", "bfloat16"):
        g = torch.Generator(device="cuda").manual_seed(1)
        dt = getattr(torch, dtype)
        H = torch.randn(N, D, generator=g, device="cuda").to(dt)
        W = (torch.randn(V, D, generator=g, device="cuda") / 8).to(dt)
        y = torch.randint(0, V, (N,), generator=g, device="cuda")
        bias = torch.zeros(V, device="cuda", dtype=dt)
        lp = -pkg.class_loss(H, W, y, bias=bias, grads=False).row_loss
        A = torch.randn(N, generator=g, device="cuda")
        A[N // 2:] *= 1000
        whole = pkg.policy_loss(H, W, y, lp, A, bias=bias, mean=False).check()
        parts = [pkg.policy_loss(H[i:i + 1000], W, y[i:i + 1000], lp[i:i + 1000], A[i:i + 1000], bias=bias, mean=False).check() for i in range(0, N, 1000)]
        eps = torch.finfo(dt).eps
        for name in ("dW", "db"):
            got, want = getattr(whole, name).double(), sum(getattr(p, name).double() for p in parts)
            # each part is rounded to the type, and so is the whole; G's rounding differs where the scale does
            size = sum(getattr(p, name).double().abs() for p in parts) + got.abs()
            norm = float((got - want).norm()) / float(size.norm())
            assert norm <= eps, (dtype, name, norm)
        got, want = whole.dH.double(), torch.cat([p.dH for p in parts]).double()
        # Rows of small coefficients in fp16: the largest coefficient c of a block is brought to 2^14 at least, where half of fp16's smallest step is 2^-25 / 2^14 = 2^-39 of c for every class (of either side, so twice), which a
        # row of dH sums over |W|; and dH itself is rounded to half of the smallest step, 2^-25, on either side.
        floor = 2 * (2.0 ** -39 * float(A.abs().max()) * float(W.double().abs().sum(0).norm()) + 2.0 ** -25 * math.sqrt(D)) if dtype == "float16" else 0.0
        over = (got - want).norm(dim=1) - 2 * eps * want.norm(dim=1) - floor
        assert float(over.max()) <= 1e-30, (dtype, float(over.max()))
        assert torch.equal(whole.logp, torch.cat([p.logp for p in parts]))


@gpu
def test_gradient_against_differences():
    """Along random directions of H, W and the bias: central differences of the loss in 64 bits (off by 1e-7 of it at a step of 1e-4), away from the borders."""
    import torch
    s = make(50, 40, 60, "float32", 8, bias=True, weights=True, ignored=0.2)
    got = pkg.policy_loss(**s).check()
    g = torch.Generator().manual_seed(9)
    for name, key in (("dH", "H"), ("dW", "W"), ("db", "bias")):
        v = torch.randn(s[key].shape, generator=g, dtype=torch.float64).cuda()
        v = v / v.norm()
        at = []
        for e in (1e-4, -1e-4):
            t = {k: (x.double() + e * v if k == key else x.double() if k in ("H", "W", "bias") else x) for k, x in s.items()}
            has = s["actions"] >= 0
            z = torch.where(has[:, None], t["H"], 0.0) @ t["W"].t() + t["bias"]
            lp = z.log_softmax(1).gather(1, s["actions"].clamp(min=0).long()[:, None])[:, 0]
            r, A, x = torch.exp(lp - s["old_logp"]), s["advantages"].double(), s["ref_logp"].double() - lp
            l = -torch.minimum(r * A, r.clamp(0.8, 1.28) * A) + 0.1 * (torch.expm1(x) - x)
            at.append(float(torch.where(has, s["row_weights"].double() * l, 0.0).sum() / has.sum()))
        want, have = (at[0] - at[1]) / 2e-4, getattr(got, name).double() * v
        assert abs(float(have.sum()) - want) <= 5e-6 * float(have.abs().sum()), (name, float(have.sum()), want)


@gpu
def test_actions_that_are_no_class_and_rows_that_do_not_count():
    import torch
    s = make(100, 32, 50, "bfloat16", 10)
    want = pkg.policy_loss(**s, mean=False)
    bad = dict(s, actions=s["actions"].clone())
    bad["actions"][3] = 50
    r = pkg.policy_loss(**bad, mean=False)
    assert bool(r.loss.isnan()) and bool(r.row_loss[3].isnan()) and int(r.row_loss.isnan().sum()) == 1 and all(bool(t.isfinite().all()) for t in (r.dH, r.dW)) and not r.dH[3].any()
    with pytest.raises(GadError) as e:
        r.check()
    assert e.value.code == -6
    gone = dict(s, actions=s["actions"].clone())
    gone["actions"][3] = -1
    r = pkg.policy_loss(**gone, mean=False).check()
    keep = torch.arange(100, device="cuda") != 3
    assert torch.equal(r.row_loss[keep], want.row_loss[keep]) and r.row_loss[3] == 0 and r.logp[3] == 0
    none = dict(s, actions=torch.full_like(s["actions"], -1))
    r = pkg.policy_loss(**none).check()
    assert r.loss.item() == 0 and not r.dH.any() and not r.dW.any() and not r.logp.any()


@gpu
def test_equal_calls_streams_and_graphs():
    import torch
    s = make(300, 96, 1000, "bfloat16", 11, bias=True)
    want = pkg.policy_loss(**s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [pkg.policy_loss(**s, stream=t) for t in streams * 3]
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for r in got for u, v in zip(r, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pkg.policy_loss(**s)
    for t in out:
        t.fill_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(out, want))


@gpu
def test_no_rows_and_refusals_of_tensors():
    import torch
    W = torch.ones(10, 16, device="cuda")
    none = torch.empty(0, device="cuda")
    r = pkg.policy_loss(torch.empty(0, 16, device="cuda"), W, torch.empty(0, dtype=torch.int32, device="cuda"), none, none).check()
    assert r.loss.item() == 0 and r.logp.shape == (0,) and not r.dW.any()
    s = make(6, 16, 10, "float32", 12)
    for change in (dict(old_logp=s["old_logp"].double()), dict(old_logp=None), dict(advantages=s["advantages"][:5]), dict(ref_logp=s["ref_logp"].cpu()), dict(actions=s["actions"].float()), dict(clip=-0.1),
                   dict(clip=(1.5, 0.2)), dict(clip=(0.2, math.nan)), dict(clip=(0.2,)), dict(clip=(0.1, 0.2, 0.3)), dict(kl_weight=-1.0), dict(kl_weight=math.inf), dict(H=s["H"].half())):
        with pytest.raises(GadError):
            pkg.policy_loss(**{**s, **change})


def test_refusals_of_the_library():
    L = head._load()
    n = ctypes.c_size_t(0)

    def ask(**k):
        a = head._PolicyLossArgs(head._ClassLossArgs(dtype=2, cols=16, classes=24, rows=5, H=256, ldh=16, W=256, ldw=16, labels=256, label_bytes=4, scale=1.0, mean=1), 256, 256, None, 0.2, 0.2, 0.0, 256)
        for f, v in k.items():
            setattr(a if hasattr(a, f) else a.head, f, v)
        return L.gad_policy_loss_workspace_bytes(ctypes.byref(a), ctypes.byref(n))
    assert ask() == 0 and n.value > 0
    for k in (dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_high=-1.0), dict(clip_high=math.nan), dict(kl_weight=-0.1), dict(kl_weight=math.inf), dict(labels=None), dict(k=3, temperature=1.0), dict(label_bytes=2), dict(cols=0)):
        assert ask(**k) == -1, k
    assert ask(clip_high=math.inf) == 0 and ask(rows=2 ** 31) == -2
    assert L.gad_policy_loss_workspace_bytes(None, ctypes.byref(n)) == -1 and L.gad_policy_loss(None, None, 0, None) == -1
