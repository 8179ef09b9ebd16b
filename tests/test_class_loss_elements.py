"""Gradients of the losses over many classes element by element, where a norm over the whole tensor would not see a lost row, tile or class.

Bounds, in the notation of test_class_loss.py (u = 2^-24, h half a step of the type, K terms of a sum in ``dot_steps(K)`` steps of the tensor core).  An element of dH or dW is a sum over
G of magnitude A = |G| |W| (|G|^T |H|).  Worst case of each part: the cut of the sum 2u a step; G's rounding h and the result's h of the result; p off by exp(2 d + ...) - 1 of
itself for logits off by d, over the magnitudes B of p and tau (they cancel in G); a probability below 2^-32 of its neighbours' largest, and a G below fp16's normal numbers, 2^-31 of the
largest coefficient together (the latter is 2^14 or more in fp16, whose half step there is 2^-25).  db is summed in fp32 before any rounding: four rows a warp, eight warps, then runs of an eighth of
the blocks of 32 rows."""
import math

import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg
from test_class_loss import U, dot_steps, make, reference

gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def compare_elements(got, ref, s, T=1.0):
    import torch
    dt = s["H"].dtype
    N, D = s["H"].shape
    V = s["W"].shape[0]
    h = torch.finfo(dt).eps / 2 if dt != torch.float32 else U
    two = "classes" in s and s["labels"] is not None and 0 < s["hard_weight"] < 1 and T != 1     # softmaxes: the sharper one's steps are longer
    code = 0.0 if dt == torch.float32 else 2.0 ** -12 * 0.6932 * (max(T, 1 / T) if two else 1.0)
    T = min(T, 1.0)                                                      # z / T is what is off, by 1 / T times as much
    logit = (dot_steps(D, dt) * 2 * U * ref["size"] + 4 * U * 1.45 * ref["zmax"]) / T
    p_rel = math.expm1(2 * logit + 2.0 ** -20 + code) + 2 * U
    assert p_rel < 0.3                                                   # (or the comparison says nothing)
    assert int(got.status.item()) == 0
    Wa, Ha = s["W"].double().abs(), torch.where(ref["counts"][:, None], s["H"].double().abs(), 0.0)
    G, B = ref["G"].abs(), ref["terms"]
    low = 2.0 ** -31 * B.sum(1).max()
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}.get(dt, 1e-37)
    for name, of, ones, K in (("dH", lambda m: m @ Wa, Wa.sum(0), V), ("dW", lambda m: m.t() @ Ha, Ha.sum(0), N), ("db", lambda m: m.sum(0), N, 0)):
        x = getattr(got, name)
        if x is None:
            continue
        want = ref[name]
        steps = dot_steps(K, dt) * 2 + 2 if K else N / 256 + 24
        tol = h * want.abs() + ((h if K else 0) + steps * U) * of(G) + p_rel * (1 + h) * of(B) + low * ones + tiny
        off = (x.double() - want).abs()
        assert bool((off <= tol).all()), "%s: element %s off by %.3g, %.3g times its bound" % (
            name, torch.nonzero(~(off <= tol))[0].tolist(), off[~(off <= tol)][0].item(), (off / tol).nan_to_num(nan=math.inf).max().item())


def offset_logits(s, offset):
    """Every logit of every row moved by `offset`, in the first column of the matrices; the others decide between the classes."""
    s["H"][:, 0] = 64.0
    s["W"][:, 0] = offset / 64.0
    return s


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("offset", [1024.0, 3000.0, -3000.0, 6016.0, 12032.0, -20032.0])
def test_gradients_at_large_logits_without_a_bias(offset, dtype):
    """The largest class's distance from itself is no more than zero, whatever its product with log2(e) is rounded to."""
    s = offset_logits(make(300, 64, 768, dtype, 3), offset)
    compare_elements(pkg.class_loss(**s), reference(**s), s)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("D", [64, 2112])
@pytest.mark.parametrize("T,offset", [(0.25, 1500.0), (0.05, 256.0), (0.01, 31.0), (0.01, -62.0), (0.004, 16.0)])
def test_gradients_at_small_temperatures_without_a_bias(T, offset, D, dtype):
    s = make(300, D, 512, dtype, 4, k=3)
    s["W"] *= T                                                          # logits / T as spread as the others
    offset_logits(s, offset)
    s.update(temperature=T, labels=None)
    compare_elements(pkg.distill_loss(**s), reference(**s), s, T)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N,D,V", [(1, 1, 1), (5, 7, 3), (130, 100, 129), (257, 64, 300), (777, 500, 2049), (300, 130, 47), (2, 4096, 1000), (16, 1032, 4099), (20, 2500, 300), (31, 3000, 515), (1300, 200, 5000),
                                   (40000, 33, 47), (2600, 500, 513)])
def test_every_element_of_the_gradients(N, D, V, dtype):
    """Odd sizes: what is left over in the last tile of every kind, tiles cut along their reduction, sums in chunks."""
    for bias, weights, ignored in ((False, False, 0.0), (True, True, 0.4)):
        s = make(N, D, V, dtype, 1, bias=bias, weights=weights, ignored=ignored)
        compare_elements(pkg.class_loss(**s), reference(**s), s)


@gpu
@pytest.mark.parametrize("N,D,V,dtype", [(60000, 40, 20011, "bfloat16"), (50000, 40, 9001, "float32")])
def test_every_element_over_blocks_of_rows(N, D, V, dtype):
    s = make(N, D, V, dtype, 4, ignored=0.1, bias=True)
    compare_elements(pkg.class_loss(**s), reference(**s), s)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N,D,V,k,T,a", [(5, 7, 3, 3, 2.0, 0.0), (130, 100, 129, 17, 2.0, 0.3), (257, 64, 300, 130, 1.0, 0.5), (40, 512, 10007, 64, 0.5, 0.25), (33, 96, 2000, 1024, 4.0, 0.1), (21, 2500, 300, 40, 1.5, 0.5),
                                         (777, 500, 2049, 9, 3.0, 0.5)])
def test_every_element_of_a_distillation(N, D, V, k, T, a, dtype):
    for bias, weights, ignored in ((False, False, 0.0), (True, True, 0.4)):
        s = make(N, D, V, dtype, 2, k=k, bias=bias, weights=weights, ignored=ignored)
        s.update(temperature=T, hard_weight=a)
        if a == 0:
            s["labels"] = None
        compare_elements(pkg.distill_loss(**s), reference(**s), s, T)


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N,D,V,pad", [(1, 9, 5, 0), (4, 72, 700, 3), (16, 72, 130, 8), (70, 120, 333, 1), (300, 257, 2049, 5), (1300, 2100, 515, 0)])
def test_what_the_outputs_held_before_is_gone_and_nothing_else_is_written(N, D, V, pad, dtype):
    """Through the C entry: outputs of NaN, a row stride beyond the columns, and a margin on either side."""
    import ctypes as C
    import torch
    from paper_2110_02987_b200 import head
    L = head._load()
    s = make(N, D, V, dtype, 6, bias=True)
    dt, margin = s["H"].dtype, 64
    want = pkg.class_loss(**s)

    def room(rows, cols, ld, t=dt):
        buf = torch.full((margin + rows * ld + margin,), math.nan, dtype=t, device="cuda")
        return buf, buf[margin:margin + rows * ld].view(rows, ld)[:, :cols]
    outs = dict(loss=room(1, 1, 1, torch.float32), row_loss=room(1, N, N, torch.float32), dH=room(N, D, D + pad), dW=room(V, D, D + pad), db=room(1, V, V))
    status = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    at = {k: v[1].data_ptr() for k, v in outs.items()}
    a = head._ClassLossArgs(dtype=head._DTYPES[dt], cols=D, classes=V, rows=N, H=s["H"].data_ptr(), ldh=D, W=s["W"].data_ptr(), ldw=D, bias=s["bias"].data_ptr(), labels=s["labels"].data_ptr(),
                            label_bytes=4, k=0, target_bytes=4, temperature=1.0, hard_weight=1.0, scale=1.0, mean=1, lddh=D + pad, lddw=D + pad, status=status[1:].data_ptr(), **at)
    need = C.c_size_t(0)
    assert L.gad_class_loss_workspace_bytes(C.byref(a), C.byref(need)) == 0
    ws = torch.full((need.value + 256,), 255, dtype=torch.uint8, device="cuda")       # (NaN in every type)
    assert L.gad_class_loss(C.byref(a), ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
    assert status.tolist() == [77, 0, 77] and bool((ws[need.value:] == 255).all())
    for name, (buf, view) in outs.items():
        assert torch.equal(view.reshape(-1), getattr(want, name).reshape(-1)), name
        assert bool(torch.isfinite(view.float()).all()) and int(torch.isnan(buf.float()).sum()) == buf.numel() - view.numel(), name


@gpu
@pytest.mark.parametrize("dtype,V", [("float16", 1 << 19), ("bfloat16", 1 << 20)])
def test_sums_over_very_many_classes_are_not_cut_short(dtype, V):
    """dH over very many classes, in so many tiles that none is cut along its reduction, where all terms have one sign and G is exact: logits of zero, so that every probability is
    2^-19 (2^-20).  The tensor core adds 16 terms at a time and cuts off at most 2u of the sum; what it adds up before the sum goes on in fp32 may cost an eighth of half a step h of the
    result, whatever V is, and the sums in fp32 one u each, of at most 2^7.  (G of the label, 1 / V - 1, is rounded to -1.)"""
    import torch
    N, D = 1280, 2048                                                    # 5 x 8 tiles for 74 pairs: two of them are not to share one
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.rand(V, D, generator=g, device="cuda", dtype=torch.float32).add_(0.5).to(dt)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    got = pkg.class_loss(torch.zeros(N, D, dtype=dt, device="cuda"), W, labels, mean=False, grads="H").check()
    total = torch.zeros(D, dtype=torch.float64, device="cuda")
    for i in range(0, V, 1 << 17):
        total += W[i:i + (1 << 17)].double().sum(0)
    hot = W[labels].double()
    want = total / V - hot
    h = torch.finfo(dt).eps / 2
    sizes = total / V + hot                                              # no partial sum is larger
    assert ((got.dH.double() - want).abs() <= h * want.abs() + (h / 8 + 2 ** 7 * U + 1 / V) * sizes).all()


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("D,sparse", [(512, False), (2048, False), (4096, False), (1433, True)])
def test_logits_that_fp32_holds_exactly_are_exact(D, sparse, dtype):
    """Whole numbers, and rows with few values (bag-of-words features): no partial sum needs more than 24 bits, so nothing is cut off and nothing is to be given back.  What is left:
    the product with log2(e), its constant, the sum of the softmax, its logarithm and the way back, a rounding of the largest number each (|z| log2(e) is below 2 |z|: 2u of it counts as 4u of |z|)."""
    import torch
    N, V = 300, 500
    g = torch.Generator().manual_seed(5)
    dt = getattr(torch, dtype)
    H = (torch.rand(N, D, generator=g) < 0.0125).float() if sparse else torch.randint(-4, 5, (N, D), generator=g).float()
    W = torch.randint(-64 if sparse else -2, 65 if sparse else 3, (V, D), generator=g).float()
    H, W = H.to(dt).cuda(), W.to(dt).cuda()
    z = H.double() @ W.double().t()
    labels = z.argmin(1)                                                 # the largest losses: twice the largest logit
    row = torch.logsumexp(z, 1) - z.min(1).values
    got = pkg.class_loss(H, W, labels, grads=False)
    most = z.abs().amax(1)
    assert ((got.row_loss.double() - row).abs() <= 3 * U * 2 * most + 2.0 ** -20).all()


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("N", [64, 512, 2048])
def test_gradients_that_are_whole_numbers_are_exact(N, dtype):
    """One class has all of the probability and another is the label: G is 1 and -1, and dW, over whole numbers, has no rounding to do; N a power of two."""
    import torch
    D, V = 72, 300
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(6)
    H = torch.zeros(N, D)
    H[torch.arange(N), torch.randint(0, D, (N,), generator=g)] = 1.0    # a value a row: column sums of at most 2^8
    bias = torch.zeros(V)
    bias[17] = 1024.0
    got = pkg.class_loss(H.to(dt).cuda(), torch.zeros(V, D, dtype=dt, device="cuda"), torch.full((N,), 290, device="cuda"), bias=bias.to(dt).cuda())
    count = H.double().sum(0)
    assert count.max() <= 2 ** 8
    want = torch.zeros(V, D, dtype=torch.float64)
    want[17], want[290] = count / N, -count / N
    assert torch.equal(got.dW.double().cpu(), want)
    assert not got.dH.any() and got.db[17].item() == 1.0 and got.db[290].item() == -1.0


def test_the_workspace_does_not_grow_with_rows_times_classes():
    """Of the rows x classes matrix 2 GB are held at most, whatever its size, and beside each logit of such a block a sixteenth of a byte to half a byte of statistics, sums and starts (16 bytes of
    statistics and 2 of starts for 128, or 64 with long rows; 4 bytes of sums of biases for 32 rows), of starts 256 MB at least; the rest goes with the rows, the classes, or their columns."""
    import ctypes as C
    from paper_2110_02987_b200 import head
    from test_class_loss import _args
    L = head._load()
    n = C.c_size_t(0)
    for dtype in (0, 1, 2):
        for rows, classes, cols, k, grads in ((16384, 1 << 24, 64, 8, False), (1 << 20, 131072, 64, 8, False), (1 << 20, 131072, 64, 8, True), (1 << 17, 1 << 22, 64, 1, True), (1 << 16, 1 << 20, 4096, 64, True),
                                              (1 << 26, 1 << 17, 8, 4, True)):
            out = 256 if grads else None
            a = _args(dtype=dtype, rows=rows, classes=classes, cols=cols, ldh=cols, ldw=cols, lddh=cols, lddw=cols, k=k, target_classes=256, teacher=256, hard_weight=0.5, temperature=2.0,
                      bias=256, dH=out, dW=out, db=out)
            assert L.gad_class_loss_workspace_bytes(C.byref(a), C.byref(n)) == 0
            parts = 6 if dtype == 0 else 2
            by_rows = rows * (parts * cols + 8 * (k + 1) + 16 + 8 + 1 + 16)
            by_classes = classes * ((parts * cols if dtype == 0 else 0) + (4 * cols + 4 if grads else 0))
            block = max(2 << 30, 256 * 16 * (classes + 256))
            assert n.value <= by_rows + by_classes + 1.5 * block + (320 << 20), (dtype, rows, classes, n.value)


@gpu
def test_targets_over_blocks_of_rows():
    s = make(60000, 40, 20011, "bfloat16", 7, k=5, ignored=0.1)
    s.update(temperature=2.0, hard_weight=0.5)
    compare_elements(pkg.distill_loss(**s), reference(**s), s, 2.0)


@gpu
@pytest.mark.parametrize("k,a", [(1, 0.5), (40, 0.0)])
def test_targets_of_many_rows_against_very_many_classes(k, a):
    """So many that where a row's targets start is looked up for a block of rows at a time; every row has all its classes in the last tile, the first, or anywhere."""
    import torch
    N, D, V = 2100, 8, (1 << 24) - 300
    g = torch.Generator(device="cuda").manual_seed(8)
    H = torch.randn(N, D, generator=g, device="cuda").bfloat16()
    W = (0.25 * torch.randn(V, D, generator=g, device="cuda")).bfloat16()
    cls = torch.randint(0, V, (N, k), generator=g, device="cuda")
    cls[::3] = V - 1 - torch.arange(k, device="cuda")
    cls[1::3] = torch.arange(k, device="cuda")
    labels = torch.randint(0, V, (N,), generator=g, device="cuda") if a else None
    teacher = torch.randn(N, k, generator=g, device="cuda")
    got = pkg.distill_loss(H, W, cls, teacher, temperature=2.0, labels=labels, hard_weight=a, grads=False).check()
    assert N * V // 64 > 1 << 28
    h, w = H.double(), W.double()
    lse, lse2 = [], []
    for i in range(0, N, 100):
        z = h[i:i + 100] @ w.t()
        lse.append(torch.logsumexp(z, 1))
        lse2.append(torch.logsumexp(z.mul_(0.5), 1))
        del z
    lse, lse2 = torch.cat(lse), torch.cat(lse2)
    q = torch.softmax(teacher.double() / 2, 1)
    zt = torch.einsum("nkd,nd->nk", w[cls], h)
    want = (1 - a) * 4 * (q * (q.log() - zt / 2 + lse2[:, None])).sum(1)
    if a:
        want += a * (lse - (w[labels] * h).sum(1))
    size = (h.abs() @ w.abs().amax(0)[:, None]).max().item()
    one = 4 * (2 * (dot_steps(D, H.dtype) * 2 * U * size + 4 * U * 1.45 * size) + 2.0 ** -20) + 16 * U * want.abs()
    assert ((got.row_loss.double() - want).abs() <= one).all()


@gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("N", [3, 12, 300])
def test_a_teacher_without_weight_adds_nothing_whatever_it_holds(N, dtype):
    """hard_weight 1: the cross entropy against the labels alone, also where the teacher's logits have no softmax."""
    import torch
    s = make(N, 64, 500, dtype, 9, k=4, bias=True)
    s["classes"].clamp_(min=0)
    s["teacher"][0], s["teacher"][1], s["teacher"][2, 1] = -math.inf, math.nan, math.inf
    want = pkg.class_loss(s["H"], s["W"], s["labels"], bias=s["bias"]).check()
    got = pkg.distill_loss(**s, temperature=3.0, hard_weight=1.0).check()
    assert all(torch.equal(u, v) for u, v in zip(got, want))
