"""Loss over many classes and distillation against the definition in 64 bits, with their gradients.

Tolerances.  u = 2^-24.  A product of two 16-bit operands is exact in fp32, and the tensor core adds 16 of them at a time to an fp32 accumulator, cutting
off at most 2u of it a time: a sum of K terms is off by at most (K / 16 + 8) 2u times the sum of magnitudes (``dot_steps``; fp32 operands in three parts: six such sums, of
which five are 2^-8 of the first, plus 2^-24 dropped: counted as K / 16 + K / 256 + 16 steps).  In norm the cut is half of that on average and the partial sums are no larger
than the result, so errors of whole tensors are held to ``steps * u`` relative to their norm.
A logit's error d goes to p as a relative error of d + (error of lse <= largest d); exp2 and the log of the sum add 2^-21 each, and the argument's rounding u |z| log2(e).
G is rounded to the operand type (half a step h = eps / 2), the result once more; the terms of a result's sum may cancel, so the first counts over their magnitudes.  With 16-bit operands a logarithm of a probability is kept in steps of 2^-11
octaves of the flatter softmax (of z, or of z / T): off by 2^-12 ln 2 of its probability, and T or 1 / T times that in the sharper one.  Everything is summed with a factor of 1, none is tuned."""
import math
import types

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from paper_2110_02987_b200 import GadError

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def dot_steps(K, dtype):
    import torch
    return K / 16 + K / 256 + 16 if dtype == torch.float32 else K / 16 + 8


def matrix(rows, cols, dtype, g, scale=1.0, pad=0, offset=0):
    import torch
    m = torch.randn(rows, cols, generator=g, dtype=torch.float64) * scale
    buf = torch.full((rows * (cols + pad) + offset,), math.nan, dtype=dtype, device="cuda")     # what lies between the rows is no number
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(m)
    return v


def make(N, D, V, dtype, seed=0, k=0, bias=False, weights=False, ignored=0.0, pad=0, offset=0, int64=False):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)
    it = torch.int64 if int64 else torch.int32
    W = matrix(V, D, dt, g, 2.0 / math.sqrt(D), pad, offset)
    H = matrix(N, D, dt, g, 1.0, pad, offset)
    labels = torch.randint(0, V, (N,), generator=g)
    drop = torch.rand(N, generator=g) < ignored
    s = dict(H=H, W=W, labels=torch.where(drop, -100, labels).to(it).cuda(),
             bias=torch.randn(V, generator=g).to(dt).cuda() if bias else None, row_weights=(torch.rand(N, generator=g) * 3 - 1).cuda() if weights else None)
    if k:
        cls = torch.randint(0, V, (N, k), generator=g)
        cls[torch.rand(N, k, generator=g) < 0.2] = -1
        cls[torch.rand(N, generator=g) < ignored] = -1
        s["classes"] = cls.to(it).cuda()
        s["teacher"] = (2 * torch.randn(N, k, generator=g)).cuda()
    return s


def reference(H, W, labels=None, bias=None, row_weights=None, classes=None, teacher=None, temperature=1.0, hard_weight=0.0, mean=True, scale=1.0):
    """The definition in 64 bits: loss, row losses, gradients, and the magnitudes that the tolerances are in."""
    import torch
    h, w = H.double(), W.double()
    N, V = h.shape[0], w.shape[0]
    z = h @ w.t()
    size = h.abs() @ w.abs().t()
    if bias is not None:
        z = z + bias.double()
    soft = classes is not None
    a = (hard_weight if labels is not None else 0.0) if soft else 1.0
    T = temperature if soft else 1.0
    f = torch.ones(N, dtype=torch.float64, device="cuda") if row_weights is None else row_weights.double()
    row = torch.zeros(N, dtype=torch.float64, device="cuda")
    G, terms = torch.zeros_like(z), torch.zeros_like(z)     # terms: magnitudes of what is subtracted in G
    counts = torch.zeros(N, dtype=torch.bool, device="cuda")
    if labels is not None and a > 0:
        y = labels.long()
        has = y >= 0
        logp = torch.log_softmax(z, 1)
        hot = torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], 1.0)
        row += torch.where(has, -a * logp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
        G += a * torch.where(has[:, None], logp.exp() - hot, 0.0)
        terms += a * torch.where(has[:, None], logp.exp() + hot, 0.0)
        counts |= has
    if soft and a < 1:
        used = classes >= 0
        has = used.any(1)
        q = torch.softmax(torch.where(used, teacher.double() / T, -math.inf), 1)
        q = torch.where(has[:, None], q, 0.0)
        Q = torch.zeros_like(z).scatter_add_(1, classes.long().clamp(min=0), q)
        logp = torch.log_softmax(z / T, 1)
        hit = torch.where(q > 0, q, 0.0) * torch.where(q > 0, logp.gather(1, classes.long().clamp(min=0)), 0.0)
        row += torch.where(has, (1 - a) * T * T * (torch.xlogy(q, q) - hit).sum(1), 0.0)
        G += (1 - a) * T * torch.where(has[:, None], logp.exp() - Q, 0.0)
        terms += (1 - a) * T * torch.where(has[:, None], logp.exp() + Q, 0.0)
        counts |= has
    n = int(counts.sum())
    factor = scale * (1.0 / n if n else 0.0) if mean else scale
    f = torch.where(counts, f, 0.0)
    G = G * (f * factor)[:, None]
    G = torch.where((f == 0)[:, None], 0.0, G)
    terms = torch.where((f == 0)[:, None], 0.0, terms * (f * factor).abs()[:, None])
    h = torch.where(counts[:, None], h, 0.0)
    return dict(loss=factor * (torch.where(counts, f * row, 0.0)).sum(), row_loss=row, dH=G @ w, dW=G.t() @ h, db=G.sum(0), G=G, size=size[counts].max().item() if n else 0.0,
                zmax=z[torch.isfinite(z)].abs().max().item(), terms=terms, weights=(f * factor).abs().sum().item(), counts=counts)


def compare(got, ref, s, T=1.0):
    import torch
    dt = s["H"].dtype
    N, D = s["H"].shape
    V = s["W"].shape[0]
    h = torch.finfo(dt).eps / 2 if dt != torch.float32 else 0.0
    logit = dot_steps(D, dt) * 2 * U * ref["size"] + 4 * U * 1.45 * ref["zmax"]
    one = (2 * logit + 2.0 ** -20) * max(1.0, T * T)                                # error of a row's loss
    assert int(got.status.item()) == 0
    assert ((got.row_loss.double() - ref["row_loss"]).abs() <= one + 2 * U * ref["row_loss"].abs() * max(1.0, T)).all()
    rows = ((ref["weights"] / max(1, int(ref["counts"].sum()))) * ref["row_loss"].abs().sum()).item()
    assert abs(got.loss.double() - ref["loss"]).item() <= one * ref["weights"] + 4 * U * max(1.0, T) * max(rows, abs(ref["loss"].item())) + 1e-30
    p_rel = 2 * logit + 2.0 ** -20 + (0.0 if dt == torch.float32 else 2.0 ** -12 * 0.6932 * max(T, 1 / T))
    Wa, Ha = s["W"].double().abs(), torch.where(ref["counts"][:, None], s["H"].double().abs(), 0.0)
    sums = dict(dH=lambda m: m @ Wa, dW=lambda m: m.t() @ Ha, db=lambda m: m.sum(0))
    for name, K in (("dH", V), ("dW", N), ("db", N)):
        x = getattr(got, name)
        if x is None:
            continue
        want = ref[name]
        assert x.dtype == dt and x.shape == want.shape
        assert torch.isfinite(x.float()).all()
        steps = dot_steps(K, dt)
        off = (x.double() - want).norm().item()
        # in norm: the result's rounding; G's, and the cut of the sum, over the magnitudes of the sum's terms (they may cancel); the logits' errors over those of p and tau, which cancel in G
        size = sums[name](ref["G"].abs()).norm().item()
        tol = max(h, U) * want.norm().item() + (max(h, U) + steps * U) * size + (p_rel + 2 * U) * sums[name](ref["terms"]).norm().item()
        sub = {torch.float16: 2.0 ** -25}.get(dt, 0.0) * math.sqrt(want.numel())   # half a step of fp16's subnormals in every element
        assert off <= tol + sub + 1e-37, (name, off, tol, want.norm().item())


CLASS_SHAPES = [(1, 1, 1), (300, 130, 1), (1, 1, 2050), (1, 64, 2), (5, 7, 3), (3, 72, 128), (130, 100, 129), (257, 64, 300), (2, 4096, 1000), (777, 500, 2049), (300, 130, 47), (1, 256, 40000), (4, 1001, 700), (8, 328, 5000), (7, 6000, 90),
                (20, 2500, 300), (130, 640, 257), (9, 64, 1 << 20),
                (5, 4096, 1000), (16, 1032, 4099), (32, 72, 33), (17, 40, 2000), (31, 3000, 515)]


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N,D,V", CLASS_SHAPES)
def test_class_loss(N, D, V, dtype):
    import torch
    for bias, weights, ignored, int64 in ((False, False, 0.0, False), (True, True, 0.4, True)):
        s = make(N, D, V, dtype, 1, bias=bias, weights=weights, ignored=ignored, int64=int64)
        got = pkg.class_loss(**s)
        compare(got, reference(**s), s)
        alone = pkg.class_loss(**s, grads=False)
        assert torch.equal(alone.loss, got.loss) and torch.equal(alone.row_loss, got.row_loss)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N,D,V,k,T,a", [(1, 64, 2, 1, 1.0, 0.0), (5, 7, 3, 3, 2.0, 0.0), (130, 100, 129, 17, 2.0, 0.3), (257, 64, 300, 130, 1.0, 0.5), (40, 512, 10007, 64, 0.5, 0.25),
                                         (33, 96, 2000, 1024, 4.0, 0.1), (64, 128, 500, 8, 3.0, 1.0),
                                         (50, 72, 600, 5, 0.25, 0.5), (6, 200, 900, 7, 2.0, 0.5), (21, 2500, 300, 40, 1.5, 0.5), (12, 328, 900, 33, 2.0, 0.3), (30, 96, 150, 60, 1.0, 0.0)])
def test_distill_loss(N, D, V, k, T, a, dtype):
    for bias, weights, ignored in ((False, False, 0.0), (True, True, 0.4)):
        s = make(N, D, V, dtype, 2, k=k, bias=bias, weights=weights, ignored=ignored)
        s.update(temperature=T, hard_weight=a)
        if a == 0:
            s["labels"] = None
        compare(pkg.distill_loss(**s), reference(**s), s, T)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("pad,offset", [(5, 0), (8, 0), (0, 1), (3, 3)])
def test_strides_and_alignments(pad, offset, dtype):
    s = make(70, 120, 333, dtype, 3, pad=pad, offset=offset, bias=True)
    ref = reference(**s)
    got = pkg.class_loss(**s)
    compare(got, ref, s)
    dense = dict(s, H=s["H"].contiguous(), W=s["W"].contiguous())
    assert all(torch_equal(u, v) for u, v in zip(got, pkg.class_loss(**dense)))


def torch_equal(u, v):
    import torch
    return torch.equal(u, v)


@gpu
@pytest.mark.parametrize("N,D,V,dtype", [(60000, 40, 20011, "bfloat16"), (50000, 40, 9001, "float32"), (2200000, 33, 47, "float16"), (40000, 33, 47, "float16"), (40000, 130, 47, "float32"),
                                         (20, 300, 30000, "bfloat16"), (1300, 200, 5000, "bfloat16")])
def test_blocks_of_rows_and_shares_of_the_reduction(N, D, V, dtype):
    """More rows than a block holds (dW and db add up over the blocks), and tiles whose reduction is shared out, with both together."""
    s = make(N, D, V, dtype, 4, ignored=0.1, bias=True)
    compare(pkg.class_loss(**s), reference(**s), s)


@gpu
@pytest.mark.parametrize("kind", ["loss", "distill"])
def test_gradients_are_differences_of_the_definition(kind):
    import torch
    s = make(6, 40, 50, "float32", 5, k=5 if kind == "distill" else 0, bias=True, weights=True, ignored=0.2)
    if kind == "distill":
        s.update(temperature=2.0, hard_weight=0.4)
    got = (pkg.distill_loss if kind == "distill" else pkg.class_loss)(**s)
    for name, grad in (("H", got.dH), ("W", got.dW), ("bias", got.db)):
        v = torch.randn(s[name].shape, generator=torch.Generator().manual_seed(9), dtype=torch.float64).cuda()
        up, down = dict(s), dict(s)
        up[name], down[name] = s[name].double() + 1e-4 * v, s[name].double() - 1e-4 * v
        diff = (reference(**up)["loss"] - reference(**down)["loss"]) / 2e-4
        # third derivatives of z are below 10 here, times 1e-8; the gradients' own error as in compare()
        assert abs(diff - (grad.double() * v).sum()) <= 1e-6 * (grad.double().norm() * v.norm() + 1)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rows_that_do_not_count_may_hold_anything(dtype):
    import torch
    s = make(50, 64, 200, dtype, 6, k=4, ignored=0.0)
    s["labels"][::3] = -1
    s["classes"][::3] = -1
    s["row_weights"] = torch.ones(50, device="cuda")
    for call, args in ((pkg.class_loss, {k: s[k] for k in ("H", "W", "labels", "row_weights")}), (pkg.distill_loss, dict(s, temperature=2.0, hard_weight=0.5))):
        clean = call(**args)
        dirty = dict(args, H=args["H"].clone(), row_weights=args["row_weights"].clone())
        dirty["H"][::6], dirty["H"][3::6] = math.nan, math.inf
        dirty["row_weights"][::3] = math.nan
        if "teacher" in args:
            dirty["teacher"] = args["teacher"].clone()
            dirty["teacher"][::3] = math.nan
        got = call(**dirty)
        assert all(torch.equal(u, v) for u, v in zip(clean, got) if u is not None)
        assert not got.dH[::3].any() and not got.row_loss[::3].any()
    none = pkg.class_loss(s["H"], s["W"], torch.full((50,), -1, device="cuda"))
    assert none.loss.item() == 0 and not none.dH.any() and not none.dW.any()


@gpu
def test_masked_classes_repeated_and_unknown_classes():
    import torch
    s = make(20, 64, 300, "bfloat16", 7, bias=True)
    s["bias"][100:] = -math.inf                                      # whole tiles without a class
    s["labels"] %= 100
    ref = reference(**s)
    got = pkg.class_loss(**s)
    compare(got, ref, s)
    assert not got.dW[100:].any() and not got.db[100:].any()
    s["labels"][3] = 200                                             # a label that is masked: infinite loss, finite gradients
    got = pkg.class_loss(**s)
    assert got.row_loss[3].item() == math.inf and got.loss.item() == math.inf and torch.isfinite(got.dH.float()).all()
    with pytest.raises(GadError):
        got.check()
    s = make(20, 64, 300, "float32", 8, k=6)
    s["classes"][:, 3] = s["classes"][:, 0]                          # the same class twice: both count
    s["teacher"][0, 1:] = -math.inf
    s["classes"][0, 0] = 7
    s.update(temperature=1.0, labels=None)
    compare(pkg.distill_loss(**s), reference(**s), s)
    s["classes"][5, 2] = 300
    got = pkg.distill_loss(**s)
    assert math.isnan(got.row_loss[5].item()) and math.isnan(got.loss.item()) and torch.isfinite(got.row_loss[:5]).all()


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("T", [0.4, 2.0, 4.0, 8.0, 20.0])
def test_classes_that_only_the_flatter_softmax_sees(T, dtype):
    """Each 128 classes have one 26 above the others: 38 octaves in the softmax of z, but exp(-26 / T) in the other one, of 127 classes."""
    import torch
    s = make(300, 64, 2050, dtype, 5, k=5)
    s["W"] *= 0.125
    s["bias"] = torch.full((2050,), -26.0, dtype=s["W"].dtype, device="cuda")
    s["bias"][17::128] = 0.0
    s.update(temperature=T, hard_weight=0.5)
    ref = reference(**s)
    got = pkg.distill_loss(**s)
    compare(got, ref, s, T)
    if T >= 4:                                # without those classes the gradient of their biases would be off by all of it
        low = torch.ones(2050, dtype=torch.bool, device="cuda")
        low[17::128] = False
        low[s["classes"].long().clamp(min=0).flatten().unique()] = False
        low[s["labels"].long().clamp(min=0).unique()] = False
        assert low.any()
        want = ref["db"][low]
        h = torch.finfo(s["W"].dtype).eps / 2
        z_err = 2 * (dot_steps(64, s["W"].dtype) * 2 * U * ref["size"] + 4 * U * 1.45 * ref["zmax"]) / T + 2.0 ** -20 + 2.0 ** -12 * 0.6932
        tiny = torch.finfo(s["W"].dtype).smallest_normal * torch.finfo(s["W"].dtype).eps / 2      # half a step of subnormals (the column sums are in fp32)
        assert ((got.db.double()[low] - want).abs() <= (h + z_err + 16 * U) * want.abs() + tiny).all()


@gpu
def test_large_logits_and_scales():
    import torch
    for dtype in ("bfloat16", "float16", "float32"):
        s = make(33, 64, 500, dtype, 9)
        s["H"] *= 40                                                   # logits of several hundred: probabilities of 0 and 1
        compare(pkg.class_loss(**s), reference(**s), s)
        s = make(33, 64, 500, dtype, 10, weights=True)
        s["row_weights"] *= 1e-4
        args = dict(s, scale=8192.0, mean=False)
        compare(pkg.class_loss(**args), reference(**args), s)


@gpu
def test_some_gradients_only_and_none():
    import torch
    s = make(100, 96, 700, "bfloat16", 11, bias=True)
    whole = pkg.class_loss(**s)
    for grads in ("H", "W", "b", "HW", ["W", "b"], False):
        got = pkg.class_loss(**s, grads=grads)
        for name, key in (("dH", "H"), ("dW", "W"), ("db", "b")):
            x = getattr(got, name)
            assert (x is not None) == bool(grads and key in grads)
            assert x is None or torch.equal(x, getattr(whole, name))
        assert torch.equal(got.loss, whole.loss) and torch.equal(got.row_loss, whole.row_loss)


@gpu
def test_equal_bits_streams_and_graphs():
    import torch
    s = make(500, 128, 3000, "float16", 12, k=9, weights=True, bias=True)
    s.update(temperature=2.0, hard_weight=0.5)
    first = pkg.distill_loss(**s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = pkg.distill_loss(**s, stream=side)
    again = pkg.distill_loss(**s)                                    # at the same time as the one in front
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(u, v) for u, v in zip(first, other)) and all(torch.equal(u, v) for u, v in zip(first, again))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = pkg.distill_loss(**s)
    fresh = make(500, 128, 3000, "float16", 13, k=9, weights=True, bias=True)
    for name in ("H", "W", "labels", "classes", "teacher", "bias", "row_weights"):
        s[name].copy_(fresh[name])
    g.replay()
    torch.cuda.synchronize()
    kept = [t.clone() for t in out]
    want = pkg.distill_loss(**s)
    assert all(torch.equal(u, v) for u, v in zip(kept, want))


@gpu
def test_rows_that_are_one_row():
    """H broadcast over the rows (a row stride of zero): dH is that of every row."""
    import torch
    for N in (5, 300):
        s = make(N, 64, 90, "bfloat16", 14)
        one = dict(s, H=s["H"][:1].expand(N, 64))
        whole = dict(s, H=one["H"].contiguous())
        assert all(torch.equal(u, v) for u, v in zip(pkg.class_loss(**one), pkg.class_loss(**whole)) if u is not None)


@gpu
def test_first_call_of_a_process_inside_a_capture():
    import subprocess
    import sys
    code = """if 1:
        import torch, paper_2110_02987_b200 as pkg
        x = torch.randn(300, 64, device="cuda").bfloat16(); W = torch.randn(500, 64, device="cuda").bfloat16()
        y = torch.randint(0, 500, (300,), device="cuda"); gamma = torch.rand(64, device="cuda")
        def step():
            h, mean, rstd = pkg.layer_norm(x, gamma)
            r = pkg.class_loss(h, W, y)
            return (r.loss, r.dW) + pkg.layer_norm_backward(r.dH, x, mean, rstd, gamma)
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


def test_kernels_of_a_chain_wait_for_the_one_in_front():
    """Every kernel that is launched to come up before the one in front of it has ended has to wait for it; a missing wait shows on the GPU only where the overlap happens."""
    import os
    import re
    from test_launch_contract import closing, kernels, CSRC
    text = "".join(open(os.path.join(CSRC, f)).read() for f in ("class_gemm.cuh", "class_loss.cu", "norm.cu"))
    text = re.sub(r"//[^\n]*", "", text)
    bodies = kernels(text)
    chained = set()
    for m in re.finditer(r"\bchain\s*\(", text):
        args = text[m.end():closing(text, m.end() - 1, "()")]
        chained |= set(re.findall(r"\b\w+_kernel\b", args))
    for name in ("grad", "kernel"):                                  # chosen beforehand
        for m in re.finditer(r"\b%s = ([^;]*);" % name, text):
            chained |= set(re.findall(r"\b(class_\w+_kernel)\b", m.group(1)))
    assert {"class_gemm_kernel", "class_grad_kernel", "class_finish_kernel", "class_few_kernel", "class_join_kernel", "class_bias_kernel", "class_pack_kernel",
            "class_rows_kernel", "class_label_rows_kernel", "norm_columns_kernel"} <= chained, chained
    for name in chained:
        assert "pdl_wait();" in bodies[name], name


@gpu
def test_no_rows():
    import torch
    W = torch.ones(10, 16, device="cuda")
    got = pkg.class_loss(torch.empty(0, 16, device="cuda"), W, torch.empty(0, dtype=torch.int32, device="cuda"), bias=torch.ones(10, device="cuda"))
    assert got.loss.item() == 0 and got.row_loss.shape == (0,) and not got.dW.any() and not got.db.any() and got.dH.shape == (0, 16) and got.status.item() == 0


@gpu
def test_a_run_of_the_operators_trains_a_student_on_what_a_gcn_answers():
    """Teacher: a trained GCN's logits per node, their largest kept.  Student: layer norm, output layer, distillation; its gradients through all of
    it against those of the definition in 64 bits."""
    import numpy as np
    import torch
    from gad_synth import make_workload, glorot_params
    w = make_workload("tiny_signal")
    with pkg.from_workload(w, glorot_params(w.dims, np.random.default_rng(0))) as g:
        for _ in range(3):
            g.train_epoch()
        logits = torch.from_numpy(g.forward()).cuda()
    k = min(3, logits.shape[1])
    teacher, classes = torch.topk(logits, k, dim=1)
    X = torch.from_numpy(np.ascontiguousarray(w.X)).cuda()
    labels = torch.from_numpy(w.labels.astype(np.int32)).cuda()
    D, V = X.shape[1], logits.shape[1]
    gen = torch.Generator().manual_seed(0)
    gamma, beta = torch.rand(D, generator=gen).cuda() + 0.5, torch.randn(D, generator=gen).cuda()
    W, b = (torch.randn(V, D, generator=gen) / math.sqrt(D)).cuda(), torch.randn(V, generator=gen).cuda()
    y, mean, rstd = pkg.layer_norm(X, gamma, beta)
    r = pkg.distill_loss(y, W, classes, teacher.contiguous(), temperature=2.0, labels=labels, hard_weight=0.5, bias=b).check()
    dx, dgamma, dbeta = pkg.layer_norm_backward(r.dH, X, mean, rstd, gamma)
    leaf = [t.double().requires_grad_() for t in (X, gamma, beta, W, b)]
    x64, g64, b64, W64, bias64 = leaf
    mu = x64.mean(1, keepdim=True)
    h = (x64 - mu) / ((x64 - mu).square().mean(1, keepdim=True) + 1e-5).sqrt() * g64 + b64
    z = h @ W64.t() + bias64
    q = torch.softmax(teacher.double() / 2, 1)
    kd = 4 * (q * (q.log() - torch.log_softmax(z / 2, 1).gather(1, classes))).sum(1).mean()
    ce = -torch.log_softmax(z, 1).gather(1, labels.long()[:, None]).mean()
    (0.5 * kd + 0.5 * ce).backward()
    for got, want in zip((dx, dgamma, dbeta, r.dW, r.db), (t.grad for t in leaf)):
        # the sums of fp32 here: D + V + N terms, 2 u a step of 16
        assert (got.double() - want).norm() <= 4 * U * ((D + V + len(labels)) / 16 + 64) * want.norm()


def _args(**kw):
    from paper_2110_02987_b200 import head
    a = dict(dtype=2, cols=64, classes=100, rows=10, H=256, ldh=64, W=256, ldw=64, bias=None, labels=256, label_bytes=4, k=0, target_classes=None, target_bytes=4,
             teacher_dtype=0, teacher=None, temperature=1.0, hard_weight=1.0, row_weights=None, scale=1.0, mean=1, loss=256, row_loss=256, dH=256, lddh=64, dW=256, lddw=64, db=None, status=256)
    a.update(kw)
    return head._ClassLossArgs(**a)


def test_refusals_on_the_host():
    import ctypes as C
    from paper_2110_02987_b200 import head
    L = head._load()
    n = C.c_size_t(0)
    assert L.gad_class_loss_workspace_bytes(C.byref(_args()), C.byref(n)) == 0 and n.value % 256 == 0 and n.value > 0
    need = n.value
    assert L.gad_class_loss_workspace_bytes(C.byref(_args(rows=0)), C.byref(n)) == 0 and n.value == 0
    nan = math.nan
    for code, kw in ((-1, dict(dtype=3)), (-1, dict(rows=-1)), (-1, dict(cols=0)), (-1, dict(classes=0)), (-1, dict(ldw=63)), (-1, dict(ldh=63)), (-1, dict(lddh=1)), (-1, dict(lddw=63)),
                     (-1, dict(label_bytes=2)), (-1, dict(k=-1)), (-2, dict(k=1025)), (-2, dict(rows=1 << 31)), (-2, dict(cols=1 << 21)), (-1, dict(scale=math.inf)), (-1, dict(scale=nan)),
                     (-1, dict(mean=2)), (-1, dict(db=256)), (-1, dict(k=2, temperature=0.0)), (-1, dict(k=2, temperature=nan)), (-1, dict(k=2, hard_weight=1.5)),
                     (-1, dict(k=2, hard_weight=nan)), (-1, dict(k=2, target_bytes=1)), (-1, dict(k=2, teacher_dtype=7))):
        assert L.gad_class_loss_workspace_bytes(C.byref(_args(**kw)), C.byref(n)) == code, kw
    # refused before anything touches a GPU
    for code, kw, ws, nws in ((-1, dict(W=None), 256, need), (-1, dict(H=None), 256, need), (-1, dict(labels=None), 256, need), (-1, dict(loss=None), 256, need), (-1, dict(row_loss=None), 256, need),
                              (-1, dict(status=None), 256, need), (-1, dict(k=2), 256, need), (-5, dict(), None, need), (-5, dict(), 256, need - 1), (-5, dict(), 128, need)):
        assert L.gad_class_loss(C.byref(_args(**kw)), ws, nws, None) == code, kw


def test_sizes_behind_32_bits_are_refused_not_cut():
    import torch
    from paper_2110_02987_b200 import head
    head._load()

    def tensor(*shape, dtype=torch.bfloat16):      # what the checks look at; nothing is allocated
        return types.SimpleNamespace(dim=lambda: 2, dtype=dtype, is_cuda=True, device="a device", shape=shape, stride=lambda: (shape[1], 1))
    many = 2 ** 32 + 8
    for call in (lambda: pkg.class_loss(tensor(4, 8), tensor(many, 8), tensor(4)), lambda: pkg.class_loss(tensor(4, many), tensor(8, many), tensor(4)),
                 lambda: pkg.distill_loss(tensor(4, 8), tensor(8, 8), tensor(4, many, dtype=torch.int32), tensor(4, many)),
                 lambda: pkg.layer_norm(tensor(1, many)), lambda: pkg.layer_norm_backward(tensor(1, many), tensor(1, many), None, None)):
        with pytest.raises(GadError) as e:
            call()
        assert e.value.code == -2


def test_refusals_of_tensors_without_a_gpu():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(GadError):
        pkg.class_loss(x, x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(GadError):
        pkg.class_loss(x, x, None)
    with pytest.raises(GadError):
        pkg.distill_loss(x, x, None, x)


@gpu
def test_refusals_of_tensors():
    import torch
    H, W = torch.zeros(4, 8, device="cuda"), torch.zeros(9, 8, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    c, t = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    for kw in (dict(H=H.half()), dict(W=W[:, :7]), dict(labels=y.float()), dict(labels=y[:3]), dict(labels=y.cpu()), dict(bias=torch.zeros(8, device="cuda")), dict(bias=torch.zeros(9, device="cuda").half()),
               dict(row_weights=torch.zeros(4, device="cuda").double()), dict(grads="HX"), dict(scale=math.nan), dict(W=W[:0]), dict(W=W[:1].expand(9, 8)), dict(H=H.t(), W=W[:, :4])):
        with pytest.raises(GadError):
            pkg.class_loss(**dict(dict(H=H, W=W, labels=y), **kw))
    for kw in (dict(classes=c[:, :2]), dict(classes=c.float()), dict(teacher=t.double()), dict(teacher=t[:, :2]), dict(temperature=0.0), dict(temperature=-1.0), dict(labels=y, hard_weight=2.0),
               dict(classes=torch.zeros(4, 1025, dtype=torch.int32, device="cuda"), teacher=torch.zeros(4, 1025, device="cuda")), dict(classes=c[:, :0], teacher=t[:, :0])):
        with pytest.raises(GadError):
            pkg.distill_loss(**dict(dict(H=H, W=W, classes=c, teacher=t), **kw))
