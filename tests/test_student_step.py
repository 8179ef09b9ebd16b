"""The operators of a student's training step in a row, as a program uses them: layer norm, gated feed-forward block, policy loss (or distillation from a trained GCN's largest
logits), the ways back, clipping, a step of gradient descent.  Gradients against those of the whole in 64 bits by autograd, the norm and the clipped values against theirs.

Tolerance, in the norm of each tensor: a product of K terms in fp32 is off by at most steps(K) of the sum of its terms' magnitudes, which is at most sqrt(K) times a sum of terms of either sign; along the longest path there
are nine products with K up to 600, the norm and the activations among them count as one more each."""
import math
import subprocess
import sys

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def tolerance(K):
    return 11 * 2 * U * (K / 16 + K / 256 + 16) * math.sqrt(K)


def student(D, F, V, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    return dict(gamma=(1 + 0.1 * r(D)).float().cuda(), beta=(0.1 * r(D)).float().cuda(), Wg=(r(F, D) / math.sqrt(D)).float().cuda(), Wu=(r(F, D) / math.sqrt(D)).float().cuda(),
                Wd=(r(D, F) / math.sqrt(F)).float().cuda(), W=(r(V, D) / math.sqrt(D)).float().cuda(), b=(0.1 * r(V)).float().cuda())


def step(X, p, loss, max_norm):
    """One pass by the library: loss, gradients by name, their norm, the clipped gradients."""
    h, mean, rstd = pkg.layer_norm(X, p["gamma"], p["beta"])
    f = pkg.gated_feed_forward(h, p["Wg"], p["Wu"], p["Wd"], save=True)
    z = X + f.y
    r = loss(z, p["W"], p["b"])
    back = pkg.gated_feed_forward_backward(r.dH, h, p["Wg"], p["Wu"], p["Wd"], f.act, f.slope, f.h)
    dX, dgamma, dbeta = pkg.layer_norm_backward(back.dx, X, mean, rstd, p["gamma"])
    grads = dict(gamma=dgamma, beta=dbeta, Wg=back.dWg, Wu=back.dWu, Wd=back.dWd, W=r.dW, b=r.db, X=dX + r.dH)
    out = {k: t.new_empty(t.shape) for k, t in grads.items()}
    norm = pkg.clip_grads(list(grads.values()), max_norm, out=list(out.values()))
    return r, f, back, grads, norm, out


def exact(X, p, loss):
    import torch
    q = {k: t.double().requires_grad_() for k, t in dict(p, X=X).items()}
    h = torch.nn.functional.layer_norm(q["X"], (X.shape[1],), q["gamma"], q["beta"], 1e-5)
    z = q["X"] + (torch.nn.functional.silu(h @ q["Wg"].t()) * (h @ q["Wu"].t())) @ q["Wd"].t()
    l = loss(z @ q["W"].t() + q["b"])
    l.backward()
    return l.detach(), {k: t.grad for k, t in q.items()}


def held(got, want, K):
    l, grads = want
    r, f, back, mine, norm, out = got
    assert int(r.status.item()) == int(f.status.item()) == int(back.status.item()) == 0
    tol = tolerance(K)
    assert abs(float(r.loss) - float(l)) <= tol * max(1.0, abs(float(l)))
    for k, t in mine.items():
        assert float((t.double() - grads[k]).norm()) <= tol * float(grads[k].norm()), k
    n = math.sqrt(sum(float(t.double().square().sum()) for t in mine.values()))
    assert abs(float(norm) - n) <= 20 * U * n
    return n


@gpu
def test_policy_step_and_descent():
    import torch
    N, D, F, V = 400, 96, 300, 600
    g = torch.Generator().manual_seed(0)
    X = torch.randn(N, D, generator=g).cuda()
    p = student(D, F, V, 1)
    y = torch.randint(0, V, (N,), generator=g).cuda()
    y[::7] = -1
    A, ref = torch.randn(N, generator=g).cuda(), None
    h, mean, rstd = pkg.layer_norm(X, p["gamma"], p["beta"])
    z = X + pkg.gated_feed_forward(h, p["Wg"], p["Wu"], p["Wd"]).y
    first = pkg.policy_loss(z, p["W"], y, torch.zeros(N, device="cuda"), A, bias=p["b"], grads=False).logp     # log-probabilities when the actions were drawn
    ref = first - 0.3
    has = y >= 0

    def exact_loss(logits):
        lp = logits.log_softmax(1).gather(1, y.clamp(min=0)[:, None])[:, 0]
        r, x = torch.exp(lp - first.double()), ref.double() - lp
        l = -torch.minimum(r * A.double(), r.clamp(0.8, 1.2) * A.double()) + 0.1 * (torch.exp(x) - x - 1)
        return torch.where(has, l, 0.0).sum() / has.sum()
    loss = lambda z, W, b: pkg.policy_loss(z, W, y, first, A, ref_logp=ref, kl_weight=0.1, bias=b)  # noqa: E731
    for _ in range(3):
        got = step(X, p, loss, 0.05)
        n = held(got, exact(X, p, exact_loss), V)
        for k, t in got[5].items():
            want = got[3][k].double() * min(1.0, 0.05 / n)
            assert float((t.double() - want).abs().max()) <= 24 * U * float(want.abs().max())
        for k in p:
            p[k] = p[k] - 0.1 * got[5][k]


@gpu
def test_distillation_step_from_a_gcn():
    import numpy as np
    import torch
    from gad_synth import make_workload, glorot_params
    w = make_workload("tiny_signal")
    with pkg.from_workload(w, glorot_params(w.dims, np.random.default_rng(0))) as g:
        for _ in range(3):
            g.train_epoch()
        logits = torch.from_numpy(g.forward()).cuda()
    k = min(3, logits.shape[1])
    teacher, classes = (t.contiguous() for t in torch.topk(logits, k))
    X = torch.from_numpy(np.ascontiguousarray(w.X)).float().cuda()
    p = student(X.shape[1], 64, logits.shape[1], 2)

    def exact_loss(z):
        q = torch.softmax(teacher.double() / 2, 1)
        return 4 * (q * (q.log() - torch.log_softmax(z / 2, 1).gather(1, classes))).sum(1).mean()
    got = step(X, p, lambda z, W, b: pkg.distill_loss(z, W, classes, teacher, temperature=2.0, bias=b), 1.0)
    held(got, exact(X, p, exact_loss), 600)


@gpu
def test_a_step_is_captured_and_replayed():
    import torch
    N, D, F, V = 300, 128, 256, 500
    g = torch.Generator().manual_seed(3)
    X, y, A = torch.randn(N, D, generator=g).cuda(), torch.randint(0, V, (N,), generator=g).cuda(), torch.randn(N, generator=g).cuda()
    p = student(D, F, V, 4)
    loss = lambda z, W, b: pkg.policy_loss(z, W, y, torch.full((N,), -6.0, device="cuda"), A, bias=b)  # noqa: E731
    want = step(X, p, loss, 0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(X, p, loss, 0.1)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0].loss, want[0].loss) and torch.equal(got[4], want[4]) and all(torch.equal(got[5][k], want[5][k]) for k in want[5])


@gpu
def test_first_calls_of_a_process_inside_a_capture():
    code = """if 1:
        import torch, paper_2110_02987_b200 as pkg
        x = torch.randn(300, 64, device="cuda").bfloat16(); W = [torch.randn(s, device="cuda").bfloat16() for s in ((96, 64), (96, 64), (64, 96), (500, 64))]
        y = torch.randint(0, 500, (300,), device="cuda"); A = torch.randn(300, device="cuda"); old = torch.full((300,), -6.0, device="cuda")
        def step():
            f = pkg.gated_feed_forward(x, *W[:3], save=True)
            few = pkg.gated_feed_forward(x[:7], *W[:3])
            r = pkg.policy_loss(f.y, W[3], y, old, A)
            s = pkg.policy_loss(f.y[:9], W[3], y[:9], old[:9], A[:9], grads=False)
            b = pkg.gated_feed_forward_backward(r.dH, x, *W[:3], f.act, f.slope, f.h)
            n = pkg.clip_grads([b.dWg, b.dWu, b.dWd, r.dW], 0.01)
            return f.y, few.y, s.logp, r.loss, n, b.dx, b.dWg, b.dWu, b.dWd, r.dW
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        g.replay(); torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        assert all(torch.equal(u, v) for u, v in zip(kept, step()))
        print("same")
    """
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=entry.ROOT)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]
