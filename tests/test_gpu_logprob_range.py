"""GPU: the gradient of log-probabilities over the whole range of logits and temperatures that the call allows: it is as near to the
formula for large logits and small temperatures as for ordinary ones."""
import math

import numpy as np
import pytest
import torch

import _train as ref
import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def check(x, targets, temp, dlogp, in_place=False, extra=0):
    """Both passes against 64 bits.  The bound does not grow with the size of the logits.

    An exponential of the gradient carries what ref.logprob says, without its term in lse.  Rows with |lse| <= 32 come from lse, which is
    m * fl(1 / T) + log(sum) and goes back through a product with T: 2 roundings of |m / T| <= 32 + log(classes), one of lse, one
    of lse * T, 2 units of log(sum) <= log(classes), and the sum's own error once more.  What is below binary32's smallest normal number may be 0,
    before and after the factor dlogp / T."""
    rows, classes = x.shape
    temp = float(np.float32(temp))                                          # what the kernel is given
    s = status()
    logp, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    srq.srq_logprob_fwd(x, targets, logp, lse, temp, device_status=s)
    _, _, _, _, rel, counts = ref.logprob(x, targets, temp)
    p = torch.softmax(x.double() / temp, 1)                                 # (an lse of 5e38 does not hold log(300) in 64 bits either)
    rel = rel + (classes / 256 + 64) * ref.ULP + ref.ULP * (128 + 4 * math.log(classes))
    d, bound = ref.dlogits(p, rel, targets, counts, dlogp.double(), 0 * dlogp.double(), temp)
    bound = bound + (dlogp.double().abs()[:, None] / temp + 1) * 2.0 ** -124
    if in_place:
        out = x.clone()
        srq.srq_logprob_bwd(out, targets, lse, dlogp, out, temp, device_status=s)
    else:
        wide = torch.full((rows, classes + extra), math.nan, dtype=x.dtype, device="cuda")
        out = wide[:, :classes]
        srq.srq_logprob_bwd(x, targets, lse, dlogp, out, temp, device_status=s)
        assert wide[:, classes:].isnan().all()
    got, half = out.double(), ref.HALF[x.dtype]
    bad = ~((got - d).abs() <= bound + half * (d.abs() + bound))
    assert not bad.any(), f"{int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {d[bad][0]}"
    return s.item()


def make(g, rows, classes, dt, offset=0.0, ties=4):
    x = torch.randn(rows, classes, generator=g, device="cuda") * 3.0 + offset
    x[::2, :ties] = 30.0 + offset                                           # several best ones of the same size
    return x.to(dt), torch.randint(0, classes, (rows,), generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [1e-6, 1e-4, 0.01, 0.3, 100.0])
def test_small_and_large_temperatures(temp, dt):
    g = torch.Generator(device="cuda").manual_seed(5)
    for rows, classes in ((9, 1000), (3, 37), (2, 131072), (2, 200001)):
        x, t, c = make(g, rows, classes, DT[dt])
        assert check(x, t, temp, c) == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1e4, -1e6, 1e6, 1e8])
def test_logits_with_a_common_offset(offset, dt):
    g = torch.Generator(device="cuda").manual_seed(6)
    for rows, classes in ((300, 513), (5, 20003)):
        x, t, c = make(g, rows, classes, DT[dt], offset)
        t[1], c[2] = -1, 0.0
        assert check(x, t, 1.0, c) == 0
        assert check(x, t, 1.0, c, in_place=True) == 0
        assert check(x, t, 1.0, c, extra=3) == 0
    assert check(torch.full((4, 300), offset, dtype=DT[dt], device="cuda"), torch.tensor([0, 7, 299, 1], device="cuda"), 1.0, torch.ones(4, device="cuda")) == 0


@pytest.mark.parametrize("rows,classes", [(1500, 70001), (40, 300001)])
def test_many_long_rows_of_both_kinds(rows, classes):
    # rows from lse and rows that are walked twice, next to one another
    g = torch.Generator(device="cuda").manual_seed(7)
    x, t, c = make(g, rows, classes, torch.bfloat16)
    x[::3] += 200.0
    assert check(x, t, 1.0, c) == 0
    assert check(x, t, 1.0, c, in_place=True) == 0


def test_an_lse_that_leaves_binary32_is_reported_and_the_gradient_is_right():
    x = torch.full((3, 300), 1e38, device="cuda")
    x[1] = 0.0
    t, c = torch.tensor([3, 4, 5], device="cuda"), torch.tensor([1.0, -2.0, 0.5], device="cuda")
    assert check(x, t, 0.2, c) == binding.ERR_NONFINITE
    s, logp = status(), torch.empty(3, device="cuda")
    srq.srq_logprob_fwd(x, t, logp, None, 0.2, device_status=s)             # nobody asks for lse: nothing is lost
    assert s.item() == 0 and (logp + math.log(300)).abs().max() < 64 * ref.ULP * 6


def test_minus_infinity_beside_large_logits():
    x = torch.full((3, 300), -math.inf, device="cuda")
    x[0, 7] = 5e7
    x[1, :2] = 1e6
    x[2, ::2] = -1e9
    t, c = torch.tensor([7, 1, 298], device="cuda"), torch.ones(3, device="cuda")
    s, logp, lse, out = status(), torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(x)
    srq.srq_logprob_fwd(x, t, logp, lse, device_status=s)
    srq.srq_logprob_bwd(x, t, lse, c, out, device_status=s)
    want = torch.zeros((3, 300), dtype=torch.float64, device="cuda")
    want[1, 0], want[1, 1] = -0.5, 0.5
    want[2, ::2] = -1 / 150
    want[2, 298] += 1
    assert s.item() == 0 and (out.double() - want).abs().max() < 300 * ref.ULP
