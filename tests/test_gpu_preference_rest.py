"""GPU: rows of the logits that belong to no answer of the preference loss, left alone or cleared."""
import math

import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import binding, lm

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,extra,offsets", [(40, 70, 0, [3, 10, 10, 20, 37]), (40, 1003, 3, [0, 10, 25]), (12, 50257, 0, [5, 6, 12]), (700, 130, 6, [1, 300, 699]),
                                                        (300, 33000, 0, [100, 150, 200]), (9, 64, 0, [4, 4, 4])])
def test_rows_of_no_answer(rows, classes, extra, offsets, dt):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, classes + extra, generator=g, device="cuda").to(DT[dt])[:, :classes]
    t = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    t[offsets[0]:offsets[-1]:7] = -1
    r = torch.randn(rows, generator=g, device="cuda")
    off = torch.tensor(offsets, device="cuda")
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[offsets[0]:offsets[-1]] = False
    x[rest], r[rest], t[rest] = math.nan, math.nan, classes + 5             # nothing of theirs is read or reported
    out = {}
    for clear in (False, True):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pair, loss, logp = torch.empty(len(offsets) // 2, device="cuda"), torch.empty(1, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        wide = torch.full((rows, classes + extra), 5.0, dtype=DT[dt], device="cuda")
        srq.srq_preference_loss(x, t, r, off, pair, loss, logp, wide[:, :classes], device_status=status, clear_rest=clear)
        assert status.item() == 0 and wide[:, classes:].eq(5).all()
        assert wide[rest, :classes].eq(0 if clear else 5).all() and logp[rest].eq(0 if clear else 9).all()
        out[clear] = [pair, loss, logp[~rest], wide[~rest]]
    for a, b in zip(out[False], out[True]):
        assert torch.equal(a, b)
    y, logp = torch.empty_like(wide)[:, :classes], torch.empty(rows, device="cuda")     # (the same pitch: the order of sums goes by alignment)
    y.copy_(x)
    srq.srq_preference_loss(y, t, r, off, pair, None, logp, y, clear_rest=True)
    assert torch.equal(y, wide[:, :classes])
    srq.srq_preference_loss(x, t, r, off, pair, None, logp, None, clear_rest=True)
    assert not logp[rest].any()


def test_no_pairs_at_all():
    for dt in DT.values():
        x = torch.full((5, 19), math.nan, dtype=dt, device="cuda")
        wide, logp, loss = torch.full((5, 24), 5.0, dtype=dt, device="cuda"), torch.full((5,), 9.0, device="cuda"), torch.ones(1, device="cuda")
        args = (x, torch.zeros(5, dtype=torch.int64, device="cuda"), logp, torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), loss, logp, wide[:, :19])
        srq.srq_preference_loss(*args)
        assert wide.eq(5).all() and logp.eq(9).all() and not loss.any()
        srq.srq_preference_loss(*args, clear_rest=True)
        assert not wide[:, :19].any() and wide[:, 19:].eq(5).all() and not logp.any()


@pytest.mark.parametrize("offsets", [[20, 50, 100], [0, 60, 90], [40, 80, 130], [70]])
def test_a_model_takes_no_gradient_from_rows_of_no_answer(offsets):
    T, V, K, F = 130, 300, 256, 384
    g = torch.Generator(device="cuda").manual_seed(1)
    pick = lambda: torch.randint(0, V, (T,), generator=g, device="cuda")  # noqa: E731
    ids, targets, ref = pick(), pick(), torch.randn(T, generator=g, device="cuda") - 5.7
    inside = torch.zeros(T, dtype=torch.bool, device="cuda")
    inside[offsets[0]:offsets[-1]] = True
    pair = torch.empty(len(offsets) // 2, device="cuda")

    def gradients(targets, offsets):
        m = lm.TokenModel(T, V, K, F, 1, embedding_scale=50.0, seed=3)
        m.initialise(0.03)
        m.forward(ids)
        loss = m.preference(targets, ref, torch.tensor(offsets, device="cuda"), pair, beta=0.5).clone()
        m.backward(ids)
        b = m.blocks[0]
        assert m.status.item() == 0
        return [loss, m.dl.dequantize(), m.dtable, m.dhead, m.dnorm, b.dwg, b.dwu, b.dwd, b.dw]
    got = gradients(targets, offsets)
    if len(offsets) == 1:
        assert not any(t.any() for t in got)
        return
    assert not got[1][~inside].any() and got[1][inside].any()
    # the same answers with rows in front and behind that do not count
    want = gradients(torch.where(inside, targets, -1), [0, offsets[1], T])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_falling_offsets_are_reported_all_the_same():
    x, t = torch.zeros((6, 64), device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")
    r, logp = torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda")
    for off in ([0, 3, 2], [-1, 2, 4], [0, 2, 7], [3, 2, 4]):
        pair, s = torch.empty(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        srq.srq_preference_loss(x, t, r, torch.tensor(off, device="cuda"), pair, None, logp, torch.empty_like(x), device_status=s, clear_rest=True)
        assert s.item() == binding.ERR_INVALID_ARG
