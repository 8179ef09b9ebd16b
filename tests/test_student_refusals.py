"""Pointers off their elements are refused on the host: a kernel that read there would fault."""
import ctypes

import pytest

import __graft_entry__ as entry
from paper_2110_02987_b200 import feed_forward as ff
from paper_2110_02987_b200 import head


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2), (2, 2)])
def test_pointers_off_their_elements(dtype, size):
    """Without a workspace, so that a call that is let through ends there (-5)."""
    L = ff._load()

    def fwd(**k):
        a = ff._ForwardArgs(dtype=dtype, cols=16, inner=24, activation=0, rows=5, ldx=17, ldwg=16, ldwu=16, ldwd=24, ldy=16, ldact=24, ldslope=24, ldh=24)     # (rows of x are copied)
        for f in ("x", "w_gate", "w_up", "w_down", "y", "act", "slope", "h", "status"):
            setattr(a, f, 256)
        for f, v in k.items():
            setattr(a, f, v)
        return L.gad_gated_feed_forward(ctypes.byref(a), None, 0, None)

    def bwd(**k):
        a = ff._BackwardArgs(dtype=dtype, cols=16, inner=24, rows=5, lddy=16, ldx=16, ldwg=16, ldwu=16, ldwd=24, ldact=24, ldslope=24, ldh=24, lddx=16, lddwg=16, lddwu=16, lddwd=24)
        for f in ("dy", "x", "w_gate", "w_up", "w_down", "act", "slope", "h", "dx", "dw_gate", "dw_up", "dw_down", "status"):
            setattr(a, f, 256)
        for f, v in k.items():
            setattr(a, f, v)
        return L.gad_gated_feed_forward_backward(ctypes.byref(a), None, 0, None)

    def policy(**k):
        h = head._ClassLossArgs(dtype=dtype, cols=16, classes=24, rows=5, H=256, ldh=16, W=256, ldw=16, labels=256, label_bytes=4, scale=1.0, mean=1, loss=256, row_loss=256, status=256)
        a = head._PolicyLossArgs(h, 256, 256, 256, 0.2, 0.2, 0.0, 256)
        for f, v in k.items():
            setattr(a, f, v)
        return L.gad_policy_loss(ctypes.byref(a), None, 0, None)
    assert fwd() == -5 and bwd() == -5 and policy() == -5
    off = 256 + size // 2
    for f in ("x", "w_gate", "w_up", "w_down", "y", "act", "slope", "h"):
        assert fwd(**{f: off}) == -1, f
        assert f == "h" and size == 2 or fwd(**{f: 256 + size}) == -5, f       # (h of 16-bit types starts on 16 bytes)
    for f in ("dy", "x", "w_gate", "w_up", "w_down", "act", "slope", "h", "dx", "dw_gate", "dw_up", "dw_down"):
        assert bwd(**{f: off}) == -1 and bwd(**{f: 256 + size}) == -5, f
    for f in ("old_logp", "advantages", "ref_logp", "logp"):
        assert policy(**{f: 258}) == -1 and policy(**{f: 260}) == -5, f
    assert fwd(status=258) == -1 and bwd(status=258) == -1
