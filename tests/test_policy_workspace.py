"""What the header says of the policy loss's workspace beside that of the loss over many classes, asked of the library on the host."""
import ctypes
import random

import pytest

import __graft_entry__ as entry
from paper_2110_02987_b200 import head


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def sizes(N, D, V, dtype, grads, bias):
    L = head._load()
    a = head._ClassLossArgs(dtype=dtype, cols=D, classes=V, rows=N, H=256, ldh=D, W=256, ldw=D, bias=256 if bias else None, labels=256, label_bytes=4, temperature=1.0, hard_weight=1.0, scale=1.0, mean=1,
                            dH=256 if grads else None, lddh=D, dW=256 if grads else None, lddw=D, db=256 if grads and bias else None)
    p = head._PolicyLossArgs(a, 256, 256, None, 0.2, 0.2, 0.0, 256)
    out = []
    for call, args in ((L.gad_class_loss_workspace_bytes, a), (L.gad_policy_loss_workspace_bytes, p)):
        n = ctypes.c_size_t(0)
        assert call(ctypes.byref(args), ctypes.byref(n)) == 0
        out.append(n.value)
    return out


def test_workspace_of_the_policy_loss():
    rng = random.Random(3)
    cases = [(13_935, 1189, 8824, 0, True, False), (8192, 1024, 8192, 0, True, True), (4096, 4096, 32_768, 0, True, False), (29_147, 2339, 378, 2, True, False), (62, 7352, 1461, 1, False, False),
             (16, 4096, 128_000, 2, False, False), (64, 4096, 1_000_000, 2, False, True), (2 ** 20, 8, 3, 0, True, True), (1, 1, 1, 0, True, True)]
    for _ in range(3000):
        cases.append((int(2 ** rng.uniform(0, 18)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 20)), rng.randrange(3), rng.random() < 0.8, rng.random() < 0.5))
    larger = 0
    for N, D, V, dtype, grads, bias in cases:
        of_class, of_policy = sizes(N, D, V, dtype, grads, bias)
        assert of_policy <= of_class + 260 * N + (1 << 20) + (320 << 20 if dtype == 0 and grads else 0), (N, D, V, dtype, grads, bias)
        larger += of_policy > of_class + N // 2 + 256
    assert larger > 0
