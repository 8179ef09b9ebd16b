"""Operators of an output head, as calls of ``paper_2110_02987_b200`` (``own``) or in plain torch operations: layer norm with its
backward pass, the softmax cross entropy of an output layer with very many classes, and distillation from a teacher's top logits.

Every case is a dict of plain values.  ``kind`` says which call it is:

  norm           ``layer_norm``: normalised rows, their means and reciprocal deviations
  norm_backward  ``layer_norm_backward``: gradients of the rows, of gamma and of beta
  loss           ``class_loss``: loss per row and in all, with ``grads`` the gradients of hidden rows, class vectors and biases
  distill        ``distill_loss``: the same against ``k`` teacher logits a row, ``hard`` of it against labels

``rows`` x ``cols`` is the matrix of hidden rows, ``pad`` what its row stride has beyond ``cols``, ``classes`` the number of classes.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # one step of serving: a few rows, launch latency is all there is
        dict(name="norm_serving", kind="norm", rows=8, cols=1024, pad=0, dtype="bf16", params32=False),
        # an ordinary batch of hidden rows
        dict(name="norm_large", kind="norm", rows=16384, cols=4096, pad=0, dtype="bf16", params32=True),
        # bag-of-words features of an odd width, rows not a multiple of 16 bytes
        dict(name="norm_odd", kind="norm", rows=20011, cols=1433, pad=0, dtype="fp32", params32=True),
        # hidden layer of a small graph
        dict(name="norm_backward_small", kind="norm_backward", rows=2708, cols=256, pad=0, dtype="fp16", params32=False),
        # the largest batch: 32 768 hidden rows, parameters in fp32 beside bf16 rows
        dict(name="norm_backward_large", kind="norm_backward", rows=32768, cols=2048, pad=0, dtype="bf16", params32=True),
        # serving: log-probability of one class for one row
        dict(name="loss_one_row", kind="loss", rows=1, cols=4096, pad=0, classes=128000, dtype="bf16", bias=False, ignored=0.0, weighted=False, grads=False),
        # nodes of a graph with a few thousand classes, in the framework's own type
        dict(name="loss_nodes_fp32", kind="loss", rows=8192, cols=256, pad=0, classes=4096, dtype="fp32", bias=True, ignored=0.3, weighted=False, grads=True),
        # an ordinary training step
        dict(name="loss_ordinary", kind="loss", rows=4096, cols=1024, pad=0, classes=32768, dtype="bf16", bias=False, ignored=0.1, weighted=False, grads=True),
        # the largest: a batch of 8192 rows against an odd number of classes
        dict(name="loss_large_odd", kind="loss", rows=8192, cols=2048, pad=0, classes=100003, dtype="bf16", bias=False, ignored=0.1, weighted=False, grads=True),
        # a small student, odd everything, rows of a wider matrix, soft and hard targets together
        dict(name="distill_odd", kind="distill", rows=777, cols=500, pad=12, classes=10007, k=17, dtype="fp16", bias=True, ignored=0.2, weighted=True, hard=0.3, temperature=2.0, grads=True),
        # distillation on the few teacher logits that are kept of each node, in the framework's own type
        dict(name="distill_nodes_fp32", kind="distill", rows=2048, cols=512, pad=0, classes=16384, k=8, dtype="fp32", bias=True, ignored=0.0, weighted=False, hard=0.0, temperature=1.0, grads=True),
        # an ordinary distillation step
        dict(name="distill_ordinary", kind="distill", rows=4096, cols=2048, pad=0, classes=50021, k=64, dtype="bf16", bias=False, ignored=0.1, weighted=False, hard=0.5, temperature=2.0, grads=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "loss", "loss", "distill", "distill"])
    dtype = rng.choice(["fp32", "fp16", "bf16"])
    pad = rng.choice([0, 0, 0, 5, 8])
    if kind.startswith("norm"):
        cols = _log_int(rng, 16, 16384)
        rows = min(_log_int(rng, 1, 65536), 32768 * 2048 // cols)
        return dict(kind=kind, rows=rows, cols=cols, pad=pad, dtype=dtype, params32=rng.random() < 0.5)
    cols, classes, rows = _log_int(rng, 32, 4096), _log_int(rng, 3, 131072), _log_int(rng, 1, 16384)
    if rng.random() < 0.5:   # widths are mostly multiples of 8
        cols = max(8, cols // 8 * 8)
    rows = max(1, min(rows, 8192 * 100003 // classes, 8192 * 100003 // classes * 2048 // cols))
    c = dict(kind=kind, rows=rows, cols=cols, pad=pad, classes=classes, dtype=dtype, bias=rng.random() < 0.5, ignored=rng.choice([0.0, 0.1, 0.5]),
             weighted=rng.random() < 0.3, grads=rng.random() < 0.8)
    if kind == "distill":
        c.update(k=min(classes, _log_int(rng, 1, 256)), hard=rng.choice([0.0, 0.3, 0.5]), temperature=rng.choice([1.0, 2.0, 0.5]))
    return c


def _matrix(g, rows, cols, pad):
    """Normal values, [rows x cols] with a row stride of cols + pad."""
    return torch.randn(rows, cols + pad, generator=g, device="cuda")[:, :cols]


def _cast(m, pad, dtype):
    out = torch.empty(m.shape[0], m.shape[1] + pad, dtype=dtype, device="cuda")[:, :m.shape[1]]
    out.copy_(m)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, rows, cols, pad = TYPES[case["dtype"]], case["rows"], case["cols"], case["pad"]
    s = dict(case=dict(case))
    if case["kind"].startswith("norm"):
        # rows with means of their own and widths of their own, as hidden rows have
        x = _matrix(g, rows, cols, pad) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda")) + torch.randn(rows, 1, generator=g, device="cuda")
        ptype = torch.float32 if case["params32"] else dtype
        s["x"] = _cast(x, pad, dtype)
        s["gamma"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(ptype)
        s["beta"] = (0.2 * torch.randn(cols, generator=g, device="cuda")).to(ptype)
        if case["kind"] == "norm_backward":
            s["dy"] = _cast(_matrix(g, rows, cols, pad), pad, dtype)
            xf = s["x"].float()
            s["mean"] = xf.mean(1)
            s["rstd"] = 1 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + EPS)
        return s
    V = case["classes"]
    W = torch.randn(V, cols, generator=g, device="cuda") * (1.5 / math.sqrt(cols))
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    # hidden rows that lean towards their class, as in the middle of training
    H = torch.randn(rows, cols, generator=g, device="cuda") + 1.5 * W[labels.long()]
    s["H"], s["W"] = _cast(H, pad, dtype), W.to(dtype)
    s["bias"] = (0.5 * torch.randn(V, generator=g, device="cuda")).to(dtype) if case["bias"] else None
    dropped = torch.rand(rows, generator=g, device="cuda") < case["ignored"]
    s["row_weights"] = torch.rand(rows, generator=g, device="cuda") + 0.5 if case["weighted"] else None
    if case["kind"] == "loss":
        s["labels"] = torch.where(dropped, -1, labels)
        return s
    # the teacher's top classes: the label's first, others behind it; some rows have fewer than k, some none
    k = case["k"]
    cls = torch.randint(0, V, (rows, k), generator=g, device="cuda", dtype=torch.int32)
    cls[:, 0] = labels
    kept = torch.randint(1, k + 1, (rows, 1), generator=g, device="cuda")
    kept = torch.where(torch.rand(rows, 1, generator=g, device="cuda") < 0.7, k, kept)
    cls = torch.where(torch.arange(k, device="cuda")[None, :] < kept, cls, -1)
    s["classes"] = torch.where(dropped[:, None], -1, cls)
    s["teacher"] = torch.sort(2 * torch.randn(rows, k, generator=g, device="cuda"), dim=1, descending=True).values
    s["labels"] = torch.where(torch.rand(rows, generator=g, device="cuda") < case["ignored"], -1, labels) if case["hard"] > 0 else None
    return s


def _run_own(s):
    import paper_2110_02987_b200 as gad
    kind = s["case"]["kind"]
    if kind == "norm":
        y, mean, rstd = gad.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS)
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "norm_backward":
        dx, dgamma, dbeta = gad.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"])
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    if kind == "loss":
        r = gad.class_loss(s["H"], s["W"], s["labels"], bias=s["bias"], row_weights=s["row_weights"], grads=s["case"]["grads"])
    else:
        r = gad.distill_loss(s["H"], s["W"], s["classes"], s["teacher"], temperature=s["case"]["temperature"], labels=s["labels"],
                             hard_weight=s["case"]["hard"], bias=s["bias"], row_weights=s["row_weights"], grads=s["case"]["grads"])
    return dict(loss=r.loss, row_loss=r.row_loss, dH=r.dH, dW=r.dW, db=r.db)


def _log_sum_exp(z):
    top = z.max(1, keepdim=True).values
    return (z - top).exp_().sum(1, keepdim=True).log_() + top


def _run_loss(s):
    case, H, W = s["case"], s["H"].float(), s["W"].float()
    N = H.shape[0]
    z = H @ W.t()
    if s["bias"] is not None:
        z += s["bias"].float()
    soft = case["kind"] == "distill"
    hard, T = (case["hard"], case["temperature"]) if soft else (1.0, 1.0)
    row = torch.zeros(N, 1, device="cuda")
    counts = torch.zeros(N, 1, dtype=torch.bool, device="cuda")
    weights = torch.ones(N, 1, device="cuda") if s["row_weights"] is None else s["row_weights"][:, None]
    if s["labels"] is not None:
        has = (s["labels"] >= 0)[:, None]
        label = s["labels"].clamp(min=0).long()[:, None]
        lse = _log_sum_exp(z)
        row += torch.where(has, hard * (lse - z.gather(1, label)), 0.0)
        counts |= has
    if soft:
        used = s["classes"] >= 0
        cls = s["classes"].clamp(min=0).long()
        some = used.any(1, keepdim=True)
        t = torch.where(used, s["teacher"] / T, -math.inf)
        t = torch.where(some, t - t.max(1, keepdim=True).values, 0.0)
        q = torch.where(used, t.exp(), 0.0)
        q = q / q.sum(1, keepdim=True).clamp(min=1e-30)
        zt = z / T
        lse_t = _log_sum_exp(zt)
        logq = torch.where(q > 0, q, 1.0).log()
        row += (1 - hard) * T * T * (q * (logq - zt.gather(1, cls) + lse_t)).sum(1, keepdim=True)
        counts |= some
    many = counts.sum().clamp(min=1)
    out = dict(loss=((weights * row).sum() / many).reshape(1), row_loss=row[:, 0], dH=None, dW=None, db=None)
    if not case["grads"]:
        return out
    f = weights / many
    if soft:
        a = torch.where(some, (1 - hard) * T * f, 0.0)
        G = zt.sub_(lse_t).exp_().mul_(a).scatter_add_(1, cls, -a * q)
        if s["labels"] is not None:
            a = torch.where(has, hard * f, 0.0)
            G += z.sub_(lse).exp_().mul_(a).scatter_add_(1, label, -a)
    else:
        a = torch.where(has, f, 0.0)
        G = z.sub_(lse).exp_().mul_(a).scatter_add_(1, label, -a)
    out["dH"] = (G @ W).to(s["H"].dtype)
    out["dW"] = (G.t() @ H).to(s["W"].dtype)
    if s["bias"] is not None:
        out["db"] = G.sum(0).to(s["bias"].dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    s = state
    kind = s["case"]["kind"]
    if kind not in ("norm", "norm_backward"):
        return _run_loss(s)
    x = s["x"].float()
    if kind == "norm":
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        y = (d * rstd * s["gamma"].float() + s["beta"].float()).to(s["x"].dtype)
        return dict(y=y, mean=mean[:, 0], rstd=rstd[:, 0])
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    g = dy * s["gamma"].float()
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd
    return dict(dx=dx.to(s["x"].dtype), dgamma=(dy * xh).sum(0).to(s["gamma"].dtype), dbeta=dy.sum(0).to(s["gamma"].dtype))


def work(case):
    e, n, d = SIZES[case["dtype"]], case["rows"], case["cols"]
    if case["kind"].startswith("norm"):
        p = 4 if case["params32"] else e
        if case["kind"] == "norm":
            return dict(bytes=2 * e * n * d + 2 * p * d + 8 * n, flops=8 * n * d)
        return dict(bytes=3 * e * n * d + 3 * p * d + 8 * n, flops=14 * n * d)
    v = case["classes"]
    targets = 8 * n * case["k"] if case["kind"] == "distill" else 4 * n
    return dict(bytes=(2 if case["grads"] else 1) * e * (n * d + v * d + (v if case["bias"] else 0)) + targets + 4 * n,
                flops=(6 if case["grads"] else 2) * n * v * d)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
        if case["kind"] == "norm":
            var, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = (var + EPS).rsqrt()
            return dict(y=torch.addcmul(beta, (x - mean[:, None]) * rstd[:, None], gamma), mean=mean, rstd=rstd)
        # as the chain rule has it: through the row's mean and variance
        dy, mean, r, D = s["dy"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None], case["cols"]
        c = x - mean
        dxh = dy * gamma
        dvar = (dxh * c).sum(1, keepdim=True) * -0.5 * r ** 3
        dx = dxh * r + dvar * 2 * c / D - (dxh * r).sum(1, keepdim=True) / D
        return dict(dx=dx, dgamma=torch.einsum("nd,nd->d", dy, c * r), dbeta=dy.sum(0))
    H, W = s["H"].double(), s["W"].double()
    N, V = H.shape[0], W.shape[0]
    b = s["bias"].double() if s["bias"] is not None else None
    soft = case["kind"] == "distill"
    hard, T = (case["hard"], case["temperature"]) if soft else (1.0, 1.0)
    w = s["row_weights"].double() if s["row_weights"] is not None else torch.ones(N, dtype=torch.float64, device="cuda")
    counted = torch.zeros(N, dtype=torch.bool, device="cuda")
    if s["labels"] is not None:
        counted |= s["labels"] >= 0
    if soft:
        counted |= (s["classes"] >= 0).any(1)
    M = max(1, int(counted.sum()))
    row = torch.zeros(N, dtype=torch.float64, device="cuda")
    grads = case["grads"]
    dH, dW = (torch.zeros_like(H), torch.zeros_like(W)) if grads else (None, None)
    db = torch.zeros(V, dtype=torch.float64, device="cuda") if grads and b is not None else None
    step = max(1, min(N, (1 << 28) // V))
    for i in range(0, N, step):   # a block of rows at a time: target distributions written out in full
        j = slice(i, min(N, i + step))
        z = H[j] @ W.t()
        if b is not None:
            z = z + b
        n = z.shape[0]
        G = torch.zeros_like(z)
        if s["labels"] is not None:
            y = s["labels"][j].long()
            at = torch.nonzero(y >= 0)[:, 0]
            logp = torch.log_softmax(z, 1)
            row[i + at] -= hard * logp[at, y[at]]
            keep = (y >= 0).double()[:, None]
            P = logp.exp_() * keep
            P[at, y[at]] -= 1
            G += hard * P
            del logp, P
        if soft:
            cls, t = s["classes"][j].long(), s["teacher"][j].double() / T
            used = cls >= 0
            has = used.any(1, keepdim=True).double()
            q = torch.nan_to_num(torch.softmax(t.masked_fill(~used, -math.inf), 1), nan=0.0)
            Q = torch.zeros_like(z).scatter_add_(1, cls.clamp(min=0), q)
            logp = torch.log_softmax(z / T, 1)
            row[i:i + n] += (1 - hard) * T * T * (torch.xlogy(q, q).sum(1) - (Q * logp).sum(1))
            G += (1 - hard) * T * (logp.exp_() * has - Q)
            del Q, logp
        if grads:
            G *= (w[j] / M)[:, None]
            dH[j] = G @ W
            dW += G.t() @ H[j]
            if db is not None:
                db += G.sum(0)
    return dict(loss=((w * row).sum() / M).reshape(1), row_loss=row, dH=dH, dW=dW, db=db)
