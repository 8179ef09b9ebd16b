"""Operators of a student's training step beside the output head, as calls of ``paper_2110_02987_b200`` (``own``) or in plain torch
operations: a gated feed-forward block with its backward pass, the clipped policy loss with a KL term over an output layer, and the
global norm and clipping of gradients.

Every case is a dict of plain values.  ``kind`` says which call it is:

  ffn           ``gated_feed_forward``: y = (act(x Wg^T) * (x Wu^T)) Wd^T, with ``save`` also what the backward pass needs
  ffn_backward  ``gated_feed_forward_backward``: gradients of x and of the three weights
  policy        ``policy_loss``: loss, loss and log-probability per row, with ``grads`` the gradients of hidden rows, class vectors and biases
  clip          ``clip_grads``: the norm over all tensors, and the tensors scaled to at most ``max_norm``

``rows`` x ``cols`` is the matrix of hidden rows, ``pad`` what its row stride has beyond ``cols``, ``inner`` the width inside the block.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"fp32": 4, "fp16": 2, "bf16": 2}
MOST_FLOPS = 12 * 16384 * 4096 * 10240     # of the largest listed case
MOST_VALUES = 750_000_000                  # gradients of the largest listed case


def listed():
    return [
        # serving: one row, reading the weights is all there is
        dict(name="ffn_one_row", kind="ffn", rows=1, cols=4096, pad=0, inner=16384, dtype="bf16", act="silu", save=False),
        # a batch of serving
        dict(name="ffn_some_rows", kind="ffn", rows=48, cols=2048, pad=0, inner=8192, dtype="bf16", act="silu", save=False),
        # odd everything, rows of a wider matrix
        dict(name="ffn_odd", kind="ffn", rows=777, cols=500, pad=12, inner=1433, dtype="fp16", act="gelu", save=False),
        # the forward pass of an ordinary training step
        dict(name="ffn_ordinary", kind="ffn", rows=8192, cols=2048, pad=0, inner=5504, dtype="bf16", act="silu", save=True),
        # nodes of a small graph, in the framework's own type
        dict(name="ffn_backward_nodes_fp32", kind="ffn_backward", rows=2708, cols=256, pad=0, inner=500, dtype="fp32", act="relu"),
        # the largest: a batch of 16 384 rows
        dict(name="ffn_backward_large", kind="ffn_backward", rows=16384, cols=4096, pad=0, inner=10240, dtype="bf16", act="silu"),
        # scoring: log-probabilities of a few rows' actions, no gradients
        dict(name="policy_score", kind="policy", rows=16, cols=4096, pad=0, classes=128000, dtype="bf16", bias=False, ignored=0.0, weighted=False, clip_low=0.2, clip_high=0.2, kl=0.05, grads=False),
        # actions on the nodes of a graph, in the framework's own type
        dict(name="policy_nodes_fp32", kind="policy", rows=8192, cols=256, pad=0, classes=2048, dtype="fp32", bias=True, ignored=0.3, weighted=True, clip_low=0.2, clip_high=0.2, kl=0.0, grads=True),
        # an ordinary step, a quarter of the rows not counting
        dict(name="policy_ordinary", kind="policy", rows=4096, cols=2048, pad=0, classes=50021, dtype="bf16", bias=False, ignored=0.25, weighted=False, clip_low=0.2, clip_high=0.28, kl=0.05, grads=True),
        # the gradients of a small student: launch latency is all there is
        dict(name="clip_small", kind="clip", tensors=12, values=150_000, layout=1, dtype="fp32", out="same", clips=True),
        # many tensors of all types, odd shapes and strides, clipped into fp32
        dict(name="clip_mixed", kind="clip", tensors=60, values=60_000_000, layout=2, dtype="mixed", out="fp32", clips=True),
        # the gradients of a large student
        dict(name="clip_large", kind="clip", tensors=63, values=MOST_VALUES, layout=3, dtype="bf16", out="same", clips=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "ffn_backward", "ffn_backward", "policy", "policy", "clip"])
    dtype = rng.choice(["fp32", "fp16", "bf16", "bf16"])
    if kind == "clip":
        values = _log_int(rng, 1000, MOST_VALUES // 2)
        return dict(kind=kind, tensors=min(values, _log_int(rng, 1, 63)), values=values, layout=rng.randrange(1 << 30), dtype=rng.choice(["fp32", "fp16", "bf16", "mixed"]),
                    out=rng.choice(["same", "fp32"]), clips=rng.random() < 0.8)
    pad = rng.choice([0, 0, 0, 5, 8])
    cols = _log_int(rng, 32, 4096)
    if rng.random() < 0.6:   # widths are mostly multiples of 8
        cols = max(8, cols // 8 * 8)
    if kind != "policy":
        inner, rows = _log_int(rng, 32, 16384), _log_int(rng, 1, 16384)
        if rng.random() < 0.6:
            inner = max(8, inner // 8 * 8)
        rows = max(1, min(rows, MOST_FLOPS // (12 * cols * inner)))
        c = dict(kind=kind, rows=rows, cols=cols, pad=pad, inner=inner, dtype=dtype, act=rng.choice(["silu", "silu", "gelu", "relu", "sigmoid"]))
        if kind == "ffn":
            c["save"] = c["act"] != "relu" and rng.random() < 0.4     # (the slope of relu jumps where the last bit of a g near 0 decides)
        return c
    classes, rows = _log_int(rng, 3, 131072), _log_int(rng, 1, 16384)
    rows = max(1, min(rows, 8192 * 100003 // classes, MOST_FLOPS // (6 * cols * classes)))
    return dict(kind=kind, rows=rows, cols=cols, pad=pad, classes=classes, dtype=dtype, bias=rng.random() < 0.5, ignored=rng.choice([0.0, 0.1, 0.5]), weighted=rng.random() < 0.3,
                clip_low=rng.choice([0.1, 0.2]), clip_high=rng.choice([0.1, 0.2, 0.28]), kl=rng.choice([0.0, 0.05, 0.1]), grads=rng.random() < 0.8)


def _layout(case):
    """The gradients' (rows, cols, pad, dtype), from the case alone: vectors and matrices, half of the matrices' rows of mixed cases in wider ones."""
    rng = random.Random(case["layout"])
    n = case["tensors"]
    # sizes over two orders of magnitude
    shares = [math.exp(rng.uniform(0.0, math.log(100.0))) for _ in range(n)]
    f = case["values"] / sum(shares)
    shapes = []
    for s in shares:
        size = max(1, int(s * f))
        mixed = case["dtype"] == "mixed"
        dtype = rng.choice(["fp32", "fp16", "bf16"]) if mixed else case["dtype"]
        if size < 256 or rng.random() < 0.3:
            shapes.append((1, size, 0, dtype))
            continue
        cols = max(1, int(math.sqrt(size) * math.exp(rng.uniform(-1.0, 1.0))))
        if not mixed and cols >= 8:
            cols = cols // 8 * 8
        shapes.append((max(1, size // cols), cols, rng.choice([0, 3, 8]) if mixed else 0, dtype))
    return shapes


def _matrix(g, rows, cols, pad):
    """Normal values, [rows x cols] with a row stride of cols + pad."""
    return torch.randn(rows, cols + pad, generator=g, device="cuda")[:, :cols]


def _cast(m, pad, dtype):
    out = torch.empty(m.shape[0], m.shape[1] + pad, dtype=dtype, device="cuda")[:, :m.shape[1]]
    out.copy_(m)
    return out


def _act(kind, g):
    """act(g) and act'(g)."""
    if kind == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if kind == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-g))
    if kind == "sigmoid":
        return s, s * (1 - s)
    return g * s, s * (1 + g * (1 - s))


def _prepare_ffn(s, g):
    case = s["case"]
    dtype, rows, cols, inner = TYPES[case["dtype"]], case["rows"], case["cols"], case["inner"]
    s["x"] = _cast(_matrix(g, rows, cols, 0), case["pad"], dtype)
    s["Wg"], s["Wu"] = ((torch.randn(inner, cols, generator=g, device="cuda") / math.sqrt(cols)).to(dtype) for _ in range(2))
    s["Wd"] = (torch.randn(cols, inner, generator=g, device="cuda") / math.sqrt(inner)).to(dtype)
    if case["kind"] == "ffn_backward":
        s["dy"] = _cast(0.1 * _matrix(g, rows, cols, 0), case["pad"], dtype)
        # what the forward pass has left: in rows of whole vectors of 8 values
        x, wide = s["x"].float(), -inner % 8
        u = x @ s["Wu"].float().t()
        a, d = _act(case["act"], x @ s["Wg"].float().t())
        s["act"], s["slope"], s["h"] = _cast(a, wide, dtype), _cast(u * d, wide, dtype), _cast(u * a, wide, dtype)


def _prepare_policy(s, g):
    case = s["case"]
    dtype, rows, cols, V = TYPES[case["dtype"]], case["rows"], case["cols"], case["classes"]
    W = torch.randn(V, cols, generator=g, device="cuda") * (1.5 / math.sqrt(cols))
    actions = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    # hidden rows that lean towards their action, as in the middle of training
    H = torch.randn(rows, cols, generator=g, device="cuda") + 1.5 * W[actions.long()]
    s["H"], s["W"] = _cast(H, case["pad"], dtype), W.to(dtype)
    s["bias"] = (0.5 * torch.randn(V, generator=g, device="cuda")).to(dtype) if case["bias"] else None
    z = s["H"].float() @ s["W"].float().t()
    if s["bias"] is not None:
        z += s["bias"].float()
    logp = z.gather(1, actions.long()[:, None])[:, 0] - _log_sum_exp(z)[:, 0]
    # the policy has moved since its actions were drawn; no ratio lies so near to a border that the last bits of a logit decide its side
    moved = 0.25 * torch.randn(rows, generator=g, device="cuda")
    for border in (math.log(1 - case["clip_low"]), math.log(1 + case["clip_high"])):
        off = moved - border
        moved = torch.where(off.abs() < 2e-3, border + torch.where(off < 0, -2e-3, 2e-3), moved)
    s["old"] = logp - moved
    s["ref"] = logp + 0.3 * torch.randn(rows, generator=g, device="cuda") if case["kl"] else None
    s["advantages"] = torch.randn(rows, generator=g, device="cuda") + 0.5     # actions that did better than their baseline, and some that did worse
    dropped = torch.rand(rows, generator=g, device="cuda") < case["ignored"]
    s["actions"] = torch.where(dropped, -1, actions)
    s["row_weights"] = torch.rand(rows, generator=g, device="cuda") + 0.5 if case["weighted"] else None


def _prepare_clip(s, g):
    case = s["case"]
    shapes = _layout(case)
    out = None if case["out"] == "same" else torch.float32
    s["grads"] = [_cast(0.02 * torch.randn(r, c, generator=g, device="cuda"), p, TYPES[t]) for r, c, p, t in shapes]
    s["out"] = [torch.empty(r, c, dtype=out or TYPES[t], device="cuda") for r, c, p, t in shapes]
    s["max_norm"] = 0.02 * math.sqrt(sum(r * c for r, c, p, t in shapes)) * (0.4 if case["clips"] else 2.5)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=dict(case))
    kind = case["kind"]
    (_prepare_clip if kind == "clip" else _prepare_policy if kind == "policy" else _prepare_ffn)(s, g)
    return s


def _run_own(s):
    import paper_2110_02987_b200 as gad
    case, kind = s["case"], s["case"]["kind"]
    if kind == "ffn":
        r = gad.gated_feed_forward(s["x"], s["Wg"], s["Wu"], s["Wd"], activation=case["act"], save=case["save"])
        return dict(y=r.y, act=r.act, slope=r.slope, h=r.h)
    if kind == "ffn_backward":
        r = gad.gated_feed_forward_backward(s["dy"], s["x"], s["Wg"], s["Wu"], s["Wd"], s["act"], s["slope"], s["h"])
        return dict(dx=r.dx, dWg=r.dWg, dWu=r.dWu, dWd=r.dWd)
    if kind == "policy":
        r = gad.policy_loss(s["H"], s["W"], s["actions"], s["old"], s["advantages"], ref_logp=s["ref"], clip=(case["clip_low"], case["clip_high"]), kl_weight=case["kl"], bias=s["bias"],
                            row_weights=s["row_weights"], grads=case["grads"])
        return dict(loss=r.loss, row_loss=r.row_loss, logp=r.logp, dH=r.dH, dW=r.dW, db=r.db)
    norm = gad.clip_grads(s["grads"], s["max_norm"], out=s["out"])
    return dict(norm=norm, grads=s["out"])


def _log_sum_exp(z):
    top = z.max(1, keepdim=True).values
    return (z - top).exp_().sum(1, keepdim=True).log_() + top


def _run_ffn(s):
    case, x, Wg, Wu, Wd = s["case"], s["x"].float(), s["Wg"].float(), s["Wu"].float(), s["Wd"].float()
    dtype = s["x"].dtype
    if case["kind"] == "ffn":
        u = x @ Wu.t()
        a, d = _act(case["act"], x @ Wg.t())
        h = a * u
        y = (h @ Wd.t()).to(dtype)
        return dict(y=y, act=a.to(dtype), slope=(u * d).to(dtype), h=h.to(dtype)) if case["save"] else dict(y=y, act=None, slope=None, h=None)
    dy = s["dy"].float()
    dh = dy @ Wd
    dg, du = dh * s["slope"].float(), dh * s["act"].float()
    return dict(dx=(dg @ Wg + du @ Wu).to(dtype), dWg=(dg.t() @ x).to(dtype), dWu=(du.t() @ x).to(dtype), dWd=(dy.t() @ s["h"].float()).to(dtype))


def _run_policy(s):
    case, H, W = s["case"], s["H"].float(), s["W"].float()
    lo, hi = case["clip_low"], case["clip_high"]
    z = H @ W.t()
    if s["bias"] is not None:
        z += s["bias"].float()
    has = s["actions"] >= 0
    action = s["actions"].clamp(min=0).long()[:, None]
    lse = _log_sum_exp(z)
    logp = torch.where(has, (z.gather(1, action) - lse)[:, 0], 0.0)
    A = s["advantages"]
    ratio = (logp - s["old"]).exp()
    plain, held = ratio * A, ratio.clamp(1 - lo, 1 + hi) * A
    row = -torch.minimum(plain, held)
    slope = torch.where(plain <= held, -plain, 0.0)
    if s["ref"] is not None:
        d = s["ref"] - logp
        row = row + case["kl"] * (d.exp() - d - 1)
        slope = slope + case["kl"] * (1 - d.exp())
    row = torch.where(has, row, 0.0)
    f = (1.0 if s["row_weights"] is None else s["row_weights"]) / has.sum().clamp(min=1)
    out = dict(loss=(f * row).sum().reshape(1), row_loss=row, logp=logp, dH=None, dW=None, db=None)
    if not case["grads"]:
        return out
    c = torch.where(has, f * slope, 0.0)[:, None]
    G = z.sub_(lse).exp_().mul_(-c).scatter_add_(1, action, c)
    out["dH"], out["dW"] = (G @ W).to(s["H"].dtype), (G.t() @ H).to(s["W"].dtype)
    if s["bias"] is not None:
        out["db"] = G.sum(0).to(s["bias"].dtype)
    return out


def _run_clip(s):
    squares = torch.stack([t.float().square().sum(dtype=torch.float64) for t in s["grads"]])
    norm = squares.sum().sqrt()
    f = (s["max_norm"] / norm).clamp(max=1.0).float()
    return dict(norm=norm.float().reshape(1), grads=[(t.float() * f).to(o.dtype) for t, o in zip(s["grads"], s["out"])])


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _run_clip(state) if kind == "clip" else _run_policy(state) if kind == "policy" else _run_ffn(state)


def work(case):
    if case["kind"] == "clip":
        shapes = _layout(case)
        n = sum(r * c for r, c, p, t in shapes)
        return dict(bytes=sum(r * c * (SIZES[t] + (4 if case["out"] == "fp32" else SIZES[t])) for r, c, p, t in shapes), flops=3 * n)
    e, n, d = SIZES[case["dtype"]], case["rows"], case["cols"]
    if case["kind"] == "policy":
        v = case["classes"]
        return dict(bytes=(2 if case["grads"] else 1) * e * (n * d + v * d + (v if case["bias"] else 0)) + (28 if case["kl"] else 24) * n, flops=(6 if case["grads"] else 2) * n * v * d)
    f = case["inner"]
    if case["kind"] == "ffn":
        return dict(bytes=e * (2 * n * d + 3 * d * f + (3 * n * f if case["save"] else 0)), flops=6 * n * d * f)
    return dict(bytes=e * (3 * n * d + 6 * d * f + 3 * n * f), flops=12 * n * d * f)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        grads = [t.double() for t in s["grads"]]
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t)) ** 2 for t in grads))
        f = min(1.0, s["max_norm"] / norm)
        return dict(norm=torch.tensor([norm], dtype=torch.float64, device="cuda"), grads=[t.mul_(f) for t in grads])
    if case["kind"] != "policy":
        x, Wg, Wu, Wd = (s[k].double() for k in ("x", "Wg", "Wu", "Wd"))
        if case["kind"] == "ffn_backward":
            dy = s["dy"].double()
            dh = torch.einsum("nd,df->nf", dy, Wd)
            dWd = torch.einsum("nd,nf->df", dy, s["h"].double())
            dg = s["slope"].double() * dh
            dx, dWg = dg @ Wg, torch.einsum("nf,nd->fd", dg, x)
            del dg
            du = dh.mul_(s["act"].double())
            return dict(dx=dx.addmm_(du, Wu), dWg=dWg, dWu=torch.einsum("nf,nd->fd", du, x), dWd=dWd)
        fun = dict(silu=torch.nn.functional.silu, gelu=torch.nn.functional.gelu, relu=torch.relu, sigmoid=torch.sigmoid)[case["act"]]
        g = torch.einsum("nd,fd->nf", x, Wg).requires_grad_()
        a = fun(g)
        u = torch.einsum("nd,fd->nf", x, Wu)
        slope = torch.autograd.grad(a, g, u)[0] if case["save"] else None      # u act'(g), by the chain rule
        a = a.detach()
        h = a * u
        return dict(y=torch.einsum("nf,df->nd", h, Wd), act=a if case["save"] else None, slope=slope, h=h if case["save"] else None)
    H, W = s["H"].double(), s["W"].double()
    N, V = H.shape[0], W.shape[0]
    b = s["bias"].double() if s["bias"] is not None else None
    lo, hi = case["clip_low"], case["clip_high"]
    w = s["row_weights"].double() if s["row_weights"] is not None else torch.ones(N, dtype=torch.float64, device="cuda")
    M = max(1, int((s["actions"] >= 0).sum()))
    row, logp = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2))
    grads = case["grads"]
    dH, dW = (torch.zeros_like(H), torch.zeros_like(W)) if grads else (None, None)
    db = torch.zeros(V, dtype=torch.float64, device="cuda") if grads and b is not None else None
    step = max(1, min(N, (1 << 28) // V))
    for i in range(0, N, step):   # a block of rows at a time
        at = i + torch.nonzero(s["actions"][i:i + step] >= 0)[:, 0]
        if not at.numel():
            continue
        y = s["actions"][at].long()
        z = H[at] @ W.t()
        if b is not None:
            z = z + b
        P = torch.log_softmax(z, 1)
        lp = P[torch.arange(at.numel(), device="cuda"), y].clone().requires_grad_()
        r, A = torch.exp(lp - s["old"][at].double()), s["advantages"][at].double()
        l = torch.where(A >= 0, -A * r.clamp(max=1 + hi), -A * r.clamp(min=1 - lo))     # the same as the smaller of the two products
        if s["ref"] is not None:
            d = s["ref"][at].double() - lp
            l = l + case["kl"] * (torch.expm1(d) - d)
        slope = torch.autograd.grad(l.sum(), lp)[0]
        row[at], logp[at] = l.detach(), lp.detach()
        if grads:
            G = P.exp_().neg_()
            G[torch.arange(at.numel(), device="cuda"), y] += 1
            G *= (slope * w[at] / M)[:, None]
            dH[at] = G @ W
            dW += G.t() @ H[at]
            if db is not None:
                db += G.sum(0)
    return dict(loss=((w * row).sum() / M).reshape(1), row_loss=row, logp=logp, dH=dH, dW=dW, db=db)
