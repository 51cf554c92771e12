"""GPU: the policy loss where an exponential leaves binary32: terms whose factor is zero are zero, and what is not finite is reported."""
import math

import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import binding

pytestmark = pytest.mark.gpu
C = 300
LOGP = -math.log(C)              # of equal logits


def call(old, adv, ref=None, x=None, rows=True, **kw):
    n = len(old)
    f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    x = torch.zeros((n, C), device="cuda") if x is None else x
    s, row, loss, logp, dx = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda"), torch.empty(1, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x)
    srq.srq_policy_loss(x, torch.full((n,), 7, device="cuda"), f(old), f(adv), torch.ones(n, device="cuda"), None if ref is None else f(ref), row if rows else None,
                        loss if rows else None, logp, dx, device_status=s, **kw)
    return s.item(), row, loss, dx


def slope(dx):
    """The gradient at logp: equal logits, dlogits at the target = c (1 - 1/C)."""
    return dx[:, 7].double() / (1 - 1 / C)


def test_no_kl_term_without_its_coefficient():
    old, adv = [LOGP, LOGP + 0.1, LOGP - 0.5], [1.0, -1.0, 0.3]
    want = call(old, adv)
    for ref in ([LOGP + 200.0, LOGP - 1e30, math.inf], [math.nan, -math.inf, 0.0]):
        got = call(old, adv, ref, kl_coef=0.0)
        assert got[0] == 0 and all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))


@pytest.mark.parametrize("clip", [0.2, math.inf])
def test_an_advantage_of_zero_with_a_ratio_beyond_binary32(clip):
    status, row, loss, dx = call([-500.0, -1000.0, LOGP], [0.0, -0.0, 0.0], clip_high=clip)
    assert status == 0 and not row.any() and not loss.any() and not dx.any()
    status, row, loss, dx = call([-500.0], [0.0], [LOGP + 0.5], kl_coef=0.2, clip_high=clip)
    assert status == 0 and abs(row.item() - 0.2 * (math.expm1(0.5) - 0.5)) < 1e-6
    assert abs(slope(dx).item() + 0.2 * math.expm1(0.5)) < 1e-6


def test_ratios_beyond_binary32():
    status, row, _, dx = call([-500.0], [1.5])                              # clipped: finite, no gradient
    assert status == 0 and abs(row.item() + 1.5 * 1.2) < 1e-6 and not dx.any()
    for adv, kw in ((-1.0, {}), (1.0, dict(clip_high=math.inf))):
        status, row, loss, _ = call([-500.0, LOGP], [adv, 0.5], **kw)
        assert status == binding.ERR_NONFINITE and row[0].isinf() and loss.isinf() and row[1].isfinite()


def test_a_row_loss_that_is_not_finite_is_reported():
    # the reference gives the class no probability: d = -inf, the loss is infinite, its slope kl is not
    status, row, loss, dx = call([LOGP], [1.0], [-math.inf], kl_coef=0.25)
    assert status == binding.ERR_NONFINITE and row.isposinf().all() and loss.isposinf().all()
    assert abs(slope(dx).item() - (0.25 - 1.0)) < 1e-5
    status, _, _, dx = call([LOGP], [1.0], [-math.inf], rows=False, kl_coef=0.25)        # nobody asks for the loss
    assert status == 0 and abs(slope(dx).item() - (0.25 - 1.0)) < 1e-5
    x = torch.zeros((1, C), device="cuda")
    x[0, 9] = math.nan                                                      # no zero factor hides it
    status, row, _, dx = call([LOGP], [0.0], x=x)
    assert status == binding.ERR_NONFINITE and row.isnan().all()
