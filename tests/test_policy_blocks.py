"""fp32 gradients of the policy loss in several blocks of rows, whose products are launched one by one, beside one block, whose products share a launch."""
import pytest

import __graft_entry__ as entry
import paper_2110_02987_b200 as pkg

gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


@gpu
@pytest.mark.parametrize("N", [1500, 2500])
def test_fp32_in_one_block_and_in_two(N):
    """Ten bytes a logit are held, 2 GiB at once: 2048 rows of 100 000 classes."""
    from test_policy_loss import make, near, reference
    s = make(N, 48, 100_000, "float32", 12, bias=True, weights=True, ignored=0.2)
    s["advantages"][N // 2:] *= 100                             # blocks with scales of their own
    near(pkg.policy_loss(**s).check(), reference(**s))
