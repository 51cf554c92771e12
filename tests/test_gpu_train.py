"""GPU: embedding, losses on the logits and the AdamW step against plain implementations (tests/_train.py) at the sizes, strides,
masks and types where they can go wrong.  The bounds are derived there."""
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def strided(t, extra):
    """t as a view with a wider pitch; the columns behind it hold NaN."""
    if not extra:
        return t.contiguous()
    wide = torch.full((t.shape[0], t.shape[1] + extra), math.nan, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def behind(view, fill_is_nan=True):
    """Whether what lies behind the columns of a strided view is still NaN."""
    base = view._base
    return base is None or bool(base[:, view.shape[1]:].isnan().all())


def near(got, want, bound, half=0.0, what=""):
    """|got - want| <= bound + half * (|want| + bound), element by element."""
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound + half * (want.abs() + bound) + 1e-300)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


# --------------------------------------------------------------------------------------------
# embedding
# --------------------------------------------------------------------------------------------
def make_ids(kind, t, v, g, dtype):
    if kind == "one":                                                       # every token the same
        ids = torch.full((t,), v // 2, device="cuda")
    elif kind == "spread":                                                  # as different as they can be
        ids = (torch.arange(t, device="cuda") * 7919) % v
    elif kind == "padded":                                                  # padding in between and at the end
        ids = torch.randint(-1, v, (t,), generator=g, device="cuda")
        ids[t - t // 3:] = -1
    elif kind == "ends":
        ids = torch.where(torch.rand(t, generator=g, device="cuda") < 0.5, 0, v - 1)
    else:                                                                   # a few ids have most of the tokens
        ids = (v ** torch.rand(t, generator=g, device="cuda").double()).long() - 1
    return ids.clamp(-1, v - 1).to(dtype)


@pytest.mark.parametrize("dt,odt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("t,v,d,extra", [(1, 1, 1, 0), (5, 7, 8, 8), (33, 100, 72, 0), (257, 1000, 136, 3), (3, 50, 2500, 0), (64, 11, 65, 0), (1000, 300, 512, 16)])
def test_embedding_forward(t, v, d, extra, dt, odt):
    g = gen(t)
    table, ids = strided(randn(g, v, d, dtype=DT[dt]), extra), make_ids("padded", t, v, g, torch.int64)
    out, s = strided(torch.full((t, d), 3.0, dtype=DT[odt], device="cuda"), extra), status()
    srq.srq_embedding_fwd(table, ids, out, 1.7, device_status=s)
    assert s.item() == 0 and torch.equal(out, ref.embed(table, ids, 1.7, DT[odt])) and behind(out)
    srq.srq_embedding_fwd(table, ids.int(), out, 1.7)
    assert torch.equal(out, ref.embed(table, ids, 1.7, DT[odt]))


def test_embedding_ids_out_of_range_give_zeros_and_a_report():
    table, out, s = torch.ones((10, 16), device="cuda"), torch.full((4, 16), 5.0, device="cuda"), status()
    ids = torch.tensor([3, 10, -7, 2 ** 40], device="cuda")
    srq.srq_embedding_fwd(table, ids, out, 2.0, device_status=s)
    assert s.item() == binding.ERR_INVALID_ARG and out[0].eq(2).all() and not out[1:].any()
    s, dt = status(), torch.full((10, 16), 5.0, device="cuda")
    srq.srq_embedding_bwd(out + 1, ids, dt, device_status=s)
    assert s.item() == binding.ERR_INVALID_ARG and dt[3].eq(3).all() and dt.count_nonzero() == 16
    s = status()
    srq.srq_embedding_bwd(out, torch.tensor([3, -1, -5, -2 ** 40], device="cuda"), dt, device_status=s)
    assert s.item() == 0
    s = status()                                                            # a table without rows
    srq.srq_embedding_fwd(torch.empty((0, 16), device="cuda"), ids[:1], out[:1], device_status=s)
    assert s.item() == binding.ERR_INVALID_ARG and not out[0].any()


CASES = [(1, 1, 1), (1, 5000, 24), (7, 3, 8), (40, 37, 130), (300, 600, 264), (513, 100, 2056), (2000, 1500, 65), (5003, 517, 136), (16384, 3000, 16)]


@pytest.mark.parametrize("kind", ["one", "spread", "padded", "ends", "few"])
@pytest.mark.parametrize("t,v,d", CASES)
def test_embedding_gradient(t, v, d, kind):
    g = gen(t + v)
    ids, s = make_ids(kind, t, v, g, torch.int64), status()
    for i, (dt, odt, extra) in enumerate([("f32", "f32", 0), ("bf16", "f32", 8), ("bf16", "bf16", 0), ("f32", "bf16", 5)]):
        dout = strided(randn(g, t, d, dtype=DT[dt]), extra)
        out = strided(torch.full((v, d), 3.0, dtype=DT[odt], device="cuda"), extra)
        srq.srq_embedding_bwd(dout, ids if i % 2 else ids.int(), out, 0.3, device_status=s)
        want, bound = ref.embed_bwd(dout, ids, v, 0.3)
        near(out, want, bound, ref.HALF[DT[odt]], f"{dt} {odt}")
        assert s.item() == 0 and behind(out)
        again = torch.empty_like(out)
        srq.srq_embedding_bwd(dout, ids, again, 0.3)
        assert torch.equal(out, again)
    # accumulating: rows without a token keep what they hold, NaN included
    dout = randn(g, t, d)
    start = randn(g, v, d)
    seen = torch.zeros(v, dtype=torch.bool, device="cuda")
    seen[ids[ids >= 0]] = True
    start[~seen] = math.nan
    out = start.clone()
    srq.srq_embedding_bwd(dout, ids, out, -2.0, accumulate=True)
    want, bound = ref.embed_bwd(dout, ids, v, -2.0)
    near(out[seen], (want + start.double())[seen], bound[seen], 2.0 ** -24, "accumulate")
    assert out[~seen].isnan().all()


@pytest.mark.parametrize("t,v", [(2049, 64), (16385, 40000), (65536, 4096), (65537, 5000), (70001, 300), (30000, 2 ** 19 + 3), (80001, 2 ** 19 + 3), (600000, 20)])
def test_embedding_gradient_of_many_tokens(t, v):
    g = gen(t)
    for kind in ("few", "padded", "one"):
        ids, s = make_ids(kind, t, v, g, torch.int64), status()
        dout, out = randn(g, t, 8, dtype=torch.bfloat16), torch.full((v, 8), 3.0, device="cuda")
        ids[5] = v + 9
        srq.srq_embedding_bwd(dout, ids, out, device_status=s)
        want, bound = ref.embed_bwd(dout, ids, v, 1.0)
        near(out, want, bound, 2.0 ** -24, kind)
        assert s.item() == binding.ERR_INVALID_ARG


def test_embedding_of_no_tokens_and_no_columns():
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    out = torch.full((9, 8), 3.0, device="cuda")
    srq.srq_embedding_bwd(torch.empty((0, 8), device="cuda"), none, out, accumulate=True)
    assert out.eq(3).all()
    srq.srq_embedding_bwd(torch.empty((0, 8), device="cuda"), none, out)
    assert not out.any()
    srq.srq_embedding_fwd(out, none, torch.empty((0, 8), device="cuda"))
    srq.srq_embedding_fwd(torch.empty((9, 0), device="cuda"), torch.tensor([3], device="cuda"), torch.empty((1, 0), device="cuda"))


def test_embedding_gradient_writes_within_its_workspace():
    t, v, d = 4000, 900, 136
    g = gen(1)
    need = srq.srq_embedding_workspace_bytes(t, v, d)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    out = torch.empty((v, d), device="cuda")
    srq.srq_embedding_bwd(randn(g, t, d), make_ids("few", t, v, g, torch.int64), out, ws=ws[:need])
    assert ws[need:].eq(0x5A).all()


# --------------------------------------------------------------------------------------------
# losses
# --------------------------------------------------------------------------------------------
def make_logits(g, rows, classes, dtype, extra, std=3.0):
    x = randn(g, rows, classes, std=std, dtype=dtype)
    targets = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    return strided(x, extra), targets


SHAPES = [(1, 1, 0), (3, 2, 1), (5, 37, 0), (64, 1000, 8), (2, 70001, 0), (40, 4097, 3), (700, 513, 0), (1, 131072, 0), (9, 32000, 0)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,extra", SHAPES)
def test_log_probabilities_and_their_gradient(rows, classes, extra, dt):
    g = gen(rows + classes)
    x, targets = make_logits(g, rows, classes, DT[dt], extra)
    if rows > 2:
        targets[1] = -100
    if classes > 8:
        x[0, 3:7] = -math.inf                                               # classes that are masked
        targets[0] = 1
    for temp, wide in ((1.0, torch.int64), (0.6, torch.int32)):
        s = status()
        logp, lse = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        srq.srq_logprob_fwd(x, targets.to(wide), logp, lse, temp, device_status=s)
        want, wlse, p, err, rel, counts = ref.logprob(x, targets, temp)
        near(logp, want, err, ref.ULP, "logp")
        near(lse, wlse, err, ref.ULP, "lse")
        dlogp = randn(g, rows)
        dlogp[-1] = 0.0
        out = strided(torch.full((rows, classes), 5.0, dtype=DT[dt], device="cuda"), extra)
        srq.srq_logprob_bwd(x, targets.to(wide), lse, dlogp, out, temp, device_status=s)
        d, bound = ref.dlogits(p, rel + err[:, None] + 4 * ref.ULP * wlse.abs()[:, None], targets, counts, dlogp.double(), 0 * dlogp.double(), temp)
        near(out, d, bound, ref.HALF[DT[dt]], "dlogits")
        assert s.item() == 0 and behind(out) and not out[-1].any()
    # in place
    y = x.clone() if not extra else strided(x, extra)
    srq.srq_logprob_bwd(y, targets, lse, dlogp, y, temp)
    assert torch.equal(y, out)


def test_log_probabilities_at_the_ends_of_the_range():
    s = status()
    x = torch.full((6, 300), -math.inf, device="cuda")
    x[0, 7] = 5.0                                                           # one class left
    x[1] = 1e38                                                             # large and equal
    x[2] = torch.linspace(-3e38, 3e38, 300, dtype=torch.float64, device="cuda").float()      # (in binary32 the spacing overflows)
    x[3, :] = -1e38
    x[4, 2], x[4, 9] = 1000.0, 999.0
    x[5] = 0.0
    targets = torch.tensor([7, 3, 299, 0, 9, -1], device="cuda")
    logp, lse = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    srq.srq_logprob_fwd(x, targets, logp, lse, device_status=s)
    want = torch.tensor([0.0, -math.log(300), 0.0, -math.log(300), -1.0 - math.log1p(math.exp(-1.0)), 0.0], dtype=torch.float64, device="cuda")
    near(logp, want, 64 * ref.ULP * 6)
    assert s.item() == 0
    # a target that is masked, a row that is masked as a whole, NaN, plus infinity: reported, the other rows are not touched by it
    for bad in ("target", "row", "nan", "inf"):
        y = torch.zeros((3, 300), device="cuda")
        if bad == "target":
            y[1, 4] = -math.inf
        elif bad == "row":
            y[1] = -math.inf
        else:
            y[1, 200] = math.nan if bad == "nan" else math.inf
        s, logp = status(), torch.empty(3, device="cuda")
        srq.srq_logprob_fwd(y, torch.tensor([4, 4, 4], device="cuda"), logp, device_status=s)
        assert s.item() == binding.ERR_NONFINITE and not logp[1].isfinite()
        near(logp[[0, 2]], torch.full((2,), -math.log(300), dtype=torch.float64, device="cuda"), 64 * ref.ULP * 6)
    # rows that do not count may hold anything
    y = torch.full((2, 300), math.nan, device="cuda")
    s, out = status(), torch.ones((2, 300), device="cuda")
    srq.srq_logprob_fwd(y, torch.tensor([-1, -5], device="cuda"), logp[:2], lse[:2], device_status=s)
    srq.srq_logprob_bwd(y, torch.tensor([-1, -5], device="cuda"), lse, torch.ones(2, device="cuda"), out, device_status=s)
    assert s.item() == 0 and not logp[:2].any() and not out.any()
    s = status()
    srq.srq_logprob_fwd(torch.zeros((1, 300), device="cuda"), torch.tensor([300], device="cuda"), logp, device_status=s)
    assert s.item() == binding.ERR_INVALID_ARG and logp[0] == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,extra", SHAPES + [(1000, 20000, 0), (700, 16391, 5), (500, 50257, 0)])      # (the last ones: many long rows)
def test_policy_loss(rows, classes, extra, dt):
    g = gen(rows * 3 + classes)
    x, targets = make_logits(g, rows, classes, DT[dt], extra, 1.5)
    temp, lo, hi, kl = 1.3, 0.2, 0.28, 0.1
    want, _, p, err, rel, counts = ref.logprob(x, targets, temp)
    old, other = (want + 0.2 * randn(g, rows).double()).float(), (want + 0.5 * randn(g, rows).double()).float()
    adv, weight = randn(g, rows), torch.rand(rows, generator=g, device="cuda") / rows
    if rows > 3:
        weight[1] = 0.0                                                     # a prompt: what it holds is not read
        old[1], adv[1], other[1], targets[2] = math.nan, math.nan, math.inf, -1
        x[1] = math.nan
        want, _, p, err, rel, counts = ref.logprob(x, targets, temp)
        counts = counts & (weight != 0)
        p[1], rel[1], err[1] = 0.0, 0.0, 0.0
    for r in (None, other):
        nan0 = lambda t: torch.where(counts, t.double(), 0.0)  # noqa: E731
        w64 = nan0(weight)
        logp64 = nan0(want)
        loss64, c = ref.policy(logp64, nan0(old), nan0(adv), w64, None if r is None else nan0(r), lo, hi, kl)
        el, ec = ref.policy_bounds(logp64, err, nan0(old), nan0(adv), w64, None if r is None else nan0(r), kl)
        # a ratio within its error of a bound of the clip may fall on either side
        rho = torch.exp(logp64 - nan0(old))
        border = torch.minimum((rho - 1 + lo).abs(), (rho - 1 - hi).abs()) <= rho * (err + 20 * ref.ULP)
        assert not border.any()                                             # none of these inputs is
        s = status()
        row, loss, logp = torch.full((rows,), 9.0, device="cuda"), torch.empty(1, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        out = strided(torch.full((rows, classes), 5.0, dtype=DT[dt], device="cuda"), extra)
        kw = dict(temperature=temp, clip_low=lo, clip_high=hi, kl_coef=kl, device_status=s)
        srq.srq_policy_loss(x, targets, old, adv, weight, r, row, loss, logp, out, **kw)
        near(logp, logp64, err, ref.ULP, "logp")
        near(row, loss64, el, ref.ULP, "row_loss")
        near(loss, loss64.sum()[None], el.sum()[None] + rows * ref.ULP * loss64.abs().sum(), ref.ULP, "loss")
        d, bound = ref.dlogits(p, rel, targets, counts, c, ec, temp)
        near(out, d, bound, ref.HALF[DT[dt]], "dlogits")
        assert s.item() == 0 and behind(out)
        # each output on its own, and in place
        y = strided(x, extra) if extra else x.clone()
        srq.srq_policy_loss(y, targets, old, adv, weight, r, dlogits=y, **kw)
        assert torch.equal(y, out)
        row2 = torch.empty_like(row)
        srq.srq_policy_loss(x, targets, old, adv, weight, r, row_loss=row2, **kw)
        assert torch.equal(row, row2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradients_whose_rows_are_aligned_otherwise_than_the_logits(dt):
    g = gen(21)
    x, targets = make_logits(g, 37, 5001, DT[dt], 0)
    dlogp = randn(g, 37)
    logp, lse = torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
    srq.srq_logprob_fwd(x, targets, logp, lse)
    want = torch.empty_like(x)
    srq.srq_logprob_bwd(x, targets, lse, dlogp, want)
    for extra in (1, 7):
        out = strided(torch.full_like(x, 5.0), extra)
        srq.srq_logprob_bwd(x, targets, lse, dlogp, out)
        assert torch.equal(out, want) and behind(out)


def test_policy_loss_clips_where_it_should():
    # logits (0, log 3): logp = log 3/4.  ratios 0.5 .. 2 through logp_old, both signs of the advantage
    x = torch.tensor([[0.0, math.log(3.0)]], device="cuda").repeat(12, 1)
    rho = torch.tensor([0.5, 0.75, 1.0, 1.15, 1.25, 2.0] * 2, device="cuda")
    old = math.log(0.75) - torch.log(rho)
    adv = torch.tensor([1.0] * 6 + [-1.0] * 6, device="cuda")
    row, out, w = torch.empty(12, device="cuda"), torch.empty((12, 2), device="cuda"), torch.ones(12, device="cuda")
    t = torch.ones(12, dtype=torch.int64, device="cuda")
    srq.srq_policy_loss(x, t, old, adv, w, None, row, None, None, out)
    clipped = torch.where(adv > 0, rho.clamp(max=1.2), rho.clamp(min=0.8))
    near(row, -clipped * adv, 1e-5)
    inside = torch.where(adv > 0, rho < 1.2, rho > 0.8)
    near(out[:, 1], torch.where(inside, -rho * adv, 0.0) * 0.25, 1e-5)
    srq.srq_policy_loss(x, t, old, adv, w, None, row, None, None, out, clip_low=math.inf, clip_high=math.inf)
    near(row, -rho * adv, 1e-5)
    near(out[:, 1], -rho * adv * 0.25, 1e-5)


def test_policy_loss_of_nothing():
    loss = torch.full((1,), 7.0, device="cuda")
    e = torch.empty(0, device="cuda")
    srq.srq_policy_loss(torch.empty((0, 50), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), e, e, e, loss=loss)
    assert loss.item() == 0
    row, s = torch.full((2,), 7.0, device="cuda"), status()
    z = torch.zeros(2, device="cuda")
    srq.srq_policy_loss(torch.empty((2, 0), device="cuda"), torch.tensor([0, -1], device="cuda"), z, z, z + 1, row_loss=row, device_status=s)
    assert not row.any() and s.item() == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,classes,extra", [([1, 1], 3, 0), ([3, 0, 0, 4], 100, 4), ([40, 33, 1, 90, 17, 300], 1003, 0), ([5, 9], 32000, 0), ([2] * 400, 50, 0)])
def test_preference_loss(lengths, classes, extra, dt):
    g = gen(sum(lengths))
    before, after = 2, 3                                                    # rows that belong to no answer
    rows = sum(lengths) + before + after
    x, targets = make_logits(g, rows, classes, DT[dt], extra, 1.5)
    if rows > 12:
        targets[5], targets[9] = -1, -100
    x[0], x[-1] = math.nan, math.nan
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]) + before, device="cuda")
    temp, beta, eps = 0.8, 0.3, 0.1
    inner = slice(before, rows - after)
    want, _, p, err, rel, counts = ref.logprob(x[inner], targets[inner], temp)
    other = torch.full((rows,), math.nan, device="cuda")
    other[inner] = (want + 0.3 * randn(g, len(want)).double()).float()
    other[inner][~counts] = math.nan
    diff = torch.where(counts, want - other[inner].double(), 0.0)
    pair64, h, c = ref.preference(diff, offsets - before, beta, eps)
    # h is off by the sums of the errors of logp; the loss and its slope (at most 1 and 1/4 per unit of h) by as much
    o = (offsets - before).tolist()
    e1 = err + 2 * ref.ULP * (want.abs() + other[inner].double().nan_to_num().abs())
    eh = beta * torch.stack([e1[a:b].sum() for a, b in zip(o, o[1:])]).view(-1, 2).sum(1) + 4 * ref.ULP * h.abs()
    ec = torch.zeros_like(c)
    for k, (a, b) in enumerate(zip(o, o[1:])):
        ec[a:b] = (eh[k // 2] / 4 + 8 * ref.ULP) * beta / len(h)
    for wide in (torch.int64, torch.int32):
        s = status()
        pair, loss, logp = torch.empty(len(h), device="cuda"), torch.empty(1, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        out = strided(torch.full((rows, classes), 5.0, dtype=DT[dt], device="cuda"), extra)
        srq.srq_preference_loss(x, targets, other, offsets.to(wide), pair, loss, logp, out, beta, eps, temp, device_status=s)
        near(logp[inner], want, err, ref.ULP, "logp")
        near(pair, pair64, eh + 8 * ref.ULP * (1 + h.abs()), ref.ULP, "pair_loss")
        near(loss, pair64.mean()[None], (eh + 8 * ref.ULP * (1 + h.abs())).mean()[None], 2 * ref.ULP, "loss")
        d, bound = ref.dlogits(p, rel, targets[inner], counts, c, ec + 8 * ref.ULP * c.abs(), temp)
        near(out[inner], d, bound, ref.HALF[DT[dt]], "dlogits")
        assert s.item() == 0 and behind(out)
        for edge in (slice(0, before), slice(rows - after, rows)):          # left as they were
            assert out[edge].eq(5).all() and logp[edge].eq(9).all()
    y = strided(x, extra) if extra else x.clone()
    srq.srq_preference_loss(y, targets, other, offsets, pair, None, logp, y, beta, eps, temp)
    assert torch.equal(y[inner], out[inner])
    pair2 = torch.empty_like(pair)
    srq.srq_preference_loss(x, targets, other, offsets, pair2, None, logp, None, beta, eps, temp)
    assert torch.equal(pair, pair2)


def test_preference_loss_of_ratios_far_apart_stays_finite():
    x = torch.zeros((2, 64), device="cuda")
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    off = torch.tensor([0, 1, 2], device="cuda")
    for gap in (2000.0, -2000.0):
        r = torch.tensor([-math.log(64) - gap, -math.log(64)], device="cuda")
        pair, logp, out, s = torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty_like(x), status()
        srq.srq_preference_loss(x, t, r, off, pair, None, logp, out, beta=1.0, device_status=s)
        assert s.item() == 0 and out.isfinite().all()
        near(pair, torch.tensor([max(0.0, -gap)], dtype=torch.float64, device="cuda"), 1e-2)


def test_preference_offsets_that_fall_are_reported():
    x, t = torch.zeros((6, 64), device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")
    r, logp = torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda")
    for off in ([0, 3, 2], [-1, 2, 4], [0, 2, 7]):
        pair, s = torch.empty(1, device="cuda"), status()
        srq.srq_preference_loss(x, t, r, torch.tensor(off, device="cuda"), pair, None, logp, torch.empty_like(x), device_status=s)
        assert s.item() == binding.ERR_INVALID_ARG and pair.item() == 0
    loss = torch.full((1,), 7.0, device="cuda")
    srq.srq_preference_loss(x, t, r, torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), loss, logp)
    assert loss.item() == 0


def test_preference_writes_within_its_workspace():
    need = srq.srq_preference_workspace_bytes(700)
    ws = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    g = gen(0)
    x, t = make_logits(g, 700, 130, torch.float32, 0)
    srq.srq_preference_loss(x, t, randn(g, 700), torch.tensor([0, 300, 700], device="cuda"), torch.empty(1, device="cuda"), None, torch.empty(700, device="cuda"),
                            torch.empty_like(x), ws=ws[:need])
    assert ws[need:].eq(0x5A).all()


# --------------------------------------------------------------------------------------------
# AdamW
# --------------------------------------------------------------------------------------------
H = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
SIZES = [1, 7, 128, 0, 129, 256, 300, 2048, 5001]


def group(sizes, pdt, gdt, bits, seed, fresh=False):
    g = gen(seed)
    out = []
    for n in sizes:
        p, gr = randn(g, n, std=0.05, dtype=pdt), randn(g, n, std=1e-2, dtype=gdt)
        m, v, ms, vs = srq.new_adam_state(p, bits)
        if not fresh and n:
            m32, v32 = randn(g, n, std=3e-3).cpu().numpy(), (randn(g, n, std=1e-2) ** 2).cpu().numpy()
            if bits == 32:
                m.copy_(torch.from_numpy(m32))
                v.copy_(torch.from_numpy(v32))
            else:
                half = np.full(n, 32767)
                c, s = ref.encode(m32, half, 448.0, 3)
                m.copy_(torch.from_numpy((c | (np.signbit(m32) * 128)).astype(np.uint8)))
                ms.copy_(torch.from_numpy(s))
                c, s = ref.encode(v32, half, 496.0, 4)
                v.copy_(torch.from_numpy(np.maximum(c, (v32 > 0)).astype(np.uint8)))
                vs.copy_(torch.from_numpy(s))
        out.append(srq.AdamTensor(p, gr, m, v, ms, vs))
    return out


def numbers(t, bits):
    """(p, g, m, v) as float32 arrays."""
    p, g = t.param.float().cpu().numpy(), t.grad.float().cpu().numpy()
    if bits == 32:
        return p, g, t.m.cpu().numpy(), t.v.cpu().numpy()
    n = len(p)
    spread = lambda s: np.repeat(s.cpu().numpy(), 128)[:n]  # noqa: E731
    c = t.m.cpu().numpy()
    m = (ref.grid_value(c & 127, 3) * np.where(c & 128, -1.0, 1.0)).astype(np.float32) * spread(t.m_step)
    return p, g, m.astype(np.float32), (ref.grid_value(t.v.cpu().numpy(), 4).astype(np.float32) * spread(t.v_step)).astype(np.float32)


def expected(t, k, bits, h, step, round_, seed, tensor_id, scale=1.0):
    """What a step makes of tensor k: (p lower, p upper, m, v or codes and steps)."""
    p, g, m, v = numbers(t, bits)
    g = (g * np.float32(scale)).astype(np.float32)
    m, v = ref.moments(m, v, g, h["beta1"], h["beta2"])
    w = ref.words(len(p), seed, tensor_id + k + (step << 32)).astype(np.int64)
    lo, hi = w & 0xFFFF, w >> 16
    x, err = ref.weight(p, m, v, h, step)
    a, b = (x - err).astype(np.float32), (x + err).astype(np.float32)
    a, b = np.nextafter(a, np.float32(-np.inf)), np.nextafter(b, np.float32(np.inf))
    if t.param.dtype == torch.bfloat16:
        if round_ == srq.SR:                    # cutting moves toward zero: the order of the two ends is that of the magnitudes
            a, b = ref.cut_bf16(a, lo), ref.cut_bf16(b, lo)
        else:
            a, b = (torch.from_numpy(q).bfloat16().float().numpy() for q in (a, b))
    if bits == 8:
        cm, sm = ref.encode(m, lo ^ hi, 448.0, 3)
        cv, sv = ref.encode(v, hi, 496.0, 4)
        cv = np.where((v > 0) & (np.repeat(sv, 128)[:len(v)] > 0), np.maximum(cv, 1), cv)
        return np.minimum(a, b), np.maximum(a, b), (cm | (np.signbit(m) * 128)).astype(np.uint8), cv.astype(np.uint8), sm, sv
    return np.minimum(a, b), np.maximum(a, b), m, v, None, None


def check_step(tensors, bits, h, step, round_, seed, tensor_id, scale=1.0, **kw):
    want = [expected(t, k, bits, h, step, round_, seed, tensor_id, scale) for k, t in enumerate(tensors)]
    s = status()
    srq.srq_adamw_step(srq.AdamTensors(tensors), **{**h, "step": step, **kw}, round=round_, seed=seed, tensor_id=tensor_id, device_status=s)
    assert s.item() == 0
    for k, (t, (a, b, m, v, sm, sv)) in enumerate(zip(tensors, want)):
        got = t.param.float().cpu().numpy()
        bad = ~((got >= a) & (got <= b))
        assert not bad.any(), f"tensor {k}: {bad.sum()} weights off, first at {np.argwhere(bad)[0]}: {got[bad][0]} outside {a[bad][0]} .. {b[bad][0]}"
        assert np.array_equal(t.m.cpu().numpy(), m), f"tensor {k}: first moment"
        assert np.array_equal(t.v.cpu().numpy(), v), f"tensor {k}: second moment"
        if bits == 8:
            assert np.array_equal(t.m_step.cpu().numpy(), sm) and np.array_equal(t.v_step.cpu().numpy(), sv), f"tensor {k}: step sizes"


@pytest.mark.parametrize("round_", [srq.SR, srq.RNE], ids=["sr", "rne"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt,gdt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_adamw_step(pdt, gdt, bits, round_):
    tensors = group(SIZES, DT[pdt], DT[gdt], bits, 3)
    check_step(tensors, bits, H, 17, round_, 5, 900)
    check_step(tensors, bits, H, 18, round_, 5, 900)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_the_first_step(bits):
    tensors = group(SIZES, torch.float32, torch.float32, bits, 4, fresh=True)
    for t in range(1, 5):
        check_step(tensors, bits, {**H, "beta1": 0.0 if t == 3 else 0.9, "beta2": 0.999}, t, srq.SR, 2 ** 40 + 1, 2 ** 33)
        for k, x in enumerate(tensors):
            x.grad.mul_(-1.5 if k % 2 else 0.01)


@pytest.mark.parametrize("count", [24, 25, 480, 481, 1000])
def test_adamw_of_many_tensors(count):
    tensors = group([(37 * k) % 400 for k in range(count)], torch.bfloat16, torch.float32, 8, 5)
    check_step(tensors, 8, H, 3, srq.SR, 1, 2 ** 32 - 30)                   # the number of the tensor carries into the upper word


def test_adamw_scalars_on_the_device_give_the_same_step():
    for bits in (32, 8):
        tensors = group(SIZES, torch.bfloat16, torch.bfloat16, bits, 6)
        lr, step, scale = torch.tensor([2e-3], device="cuda"), torch.tensor([1234], device="cuda"), torch.tensor([0.37], device="cuda")
        want = [expected(t, k, bits, {**H, "lr": float(lr.item())}, 1234, srq.SR, 5, 7, float(scale.item())) for k, t in enumerate(tensors)]
        srq.srq_adamw_step(srq.AdamTensors(tensors), **{**H, "lr": 1.0}, step=1, seed=5, tensor_id=7, lr_device=lr, step_device=step, grad_scale=scale)
        for t, (a, b, m, v, sm, sv) in zip(tensors, want):
            got = t.param.float().cpu().numpy()
            assert ((got >= a) & (got <= b)).all() and np.array_equal(t.m.cpu().numpy(), m) and np.array_equal(t.v.cpu().numpy(), v)


def test_adamw_extreme_gradients():
    # blocks without a gradient, tiny, huge, and with a spread that leaves the codes' range
    g = gen(7)
    for bits in (32, 8):
        t = group([128 * 6 + 50], torch.float32, torch.float32, bits, 8, fresh=True)[0]
        t.grad[:128] = 0
        t.grad[128:256] = 1e-25
        t.grad[256:384] = 1e17 * randn(g, 128)
        t.grad[384:512] = 10.0 ** (-12 * torch.rand(128, generator=g, device="cuda"))
        t.grad[512:640] = 0
        t.grad[530] = 3.0
        for step in (1, 2, 3):
            check_step([t], bits, {**H, "eps": 1e-6}, step, srq.SR, 9, 9)
    assert not t.v[:128].any() and bool((t.v[384:512] > 0).all()) and t.v[512:640].count_nonzero() == 1


@pytest.mark.parametrize("what", [math.nan, math.inf, 1e30])
def test_adamw_reports_what_is_not_finite(what):
    for bits in (32, 8):
        t = group([1000], torch.float32, torch.float32, bits, 9)[0]
        old = [x.clone() for x in (t.param, t.m, t.v)]
        good = t.grad.clone()
        t.grad[300] = what
        s = status()
        srq.srq_adamw_step(srq.AdamTensors([t]), **H, step=2, device_status=s)
        assert s.item() == binding.ERR_NONFINITE
        other = group([1000], torch.float32, torch.float32, bits, 9)[0]
        assert torch.equal(other.grad, good)
        srq.srq_adamw_step(srq.AdamTensors([other]), **H, step=2)
        near_by = torch.zeros(1000, dtype=torch.bool, device="cuda")
        near_by[slice(256, 384) if bits == 8 else 300] = True
        for a, b, c in zip((t.param, t.m, t.v), (other.param, other.m, other.v), old):
            assert torch.equal(a[~near_by], b[~near_by])
            if bits == 8:
                assert torch.equal(a[near_by], c[near_by])                  # left as it was
    # a factor that is not finite changes nothing
    old = [x.clone() for x in (t.param, t.m, t.v)]
    s = status()
    srq.srq_adamw_step(srq.AdamTensors([t]), **H, step=3, grad_scale=torch.tensor([math.inf], device="cuda"), device_status=s)
    assert s.item() == binding.ERR_NONFINITE and all(torch.equal(a, b) for a, b in zip(old, (t.param, t.m, t.v)))
    for kw, why in ((dict(lr_device=torch.tensor([math.nan], device="cuda")), binding.ERR_NONFINITE),
                    (dict(step_device=torch.zeros(1, dtype=torch.int64, device="cuda")), binding.ERR_INVALID_ARG)):
        s = status()
        srq.srq_adamw_step(srq.AdamTensors([t]), **H, step=3, **kw, device_status=s)
        assert s.item() == why and all(torch.equal(a, b) for a, b in zip(old, (t.param, t.m, t.v)))


def test_adamw_rounds_small_updates_with_the_right_probability():
    # an update of 1/50 of a bfloat16 unit: rounded to nearest nothing moves, stochastically the mean moves by it
    n = 1 << 16
    h = dict(lr=2.0 ** -7 / 50, beta1=0.0, beta2=0.0, eps=1e-12, weight_decay=0.0)       # u = sign of the gradient
    for round_ in (srq.RNE, srq.SR):
        t = srq.AdamTensor(torch.full((n,), 1.5, dtype=torch.bfloat16, device="cuda"), torch.full((n,), -0.25, device="cuda"), *srq.new_adam_state(torch.empty(n, device="cuda")))
        a = srq.AdamTensors([t])
        for step in range(1, 26):
            srq.srq_adamw_step(a, **h, step=step, round=round_, seed=3)
        moved = (t.param.double().mean().item() - 1.5) / (2.0 ** -7)
        # 25 steps of 1/50: half a unit; a binomial's deviation over n elements is 0.5 / 256, six of them
        assert moved == 0 if round_ == srq.RNE else abs(moved - 0.5) < 6 * 0.5 / 256


def test_adamw_leaves_what_lies_between_the_tensors_alone():
    flat = [torch.full((4096,), 7.0, device="cuda") for _ in range(4)]
    views = [(8, 1001), (1024, 5), (1536, 2000)]
    t = [srq.AdamTensor(*(f[a:a + n] for f in flat)) for a, n in views]
    srq.srq_adamw_step(srq.AdamTensors(t), **H, step=1)
    inside = torch.zeros(4096, dtype=torch.bool, device="cuda")
    for a, n in views:
        inside[a:a + n] = True
    for f in flat:
        assert f[~inside].eq(7).all()
    for f in (flat[0], flat[3]):                                            # (the first moment stays: 0.9 * 7 + 0.1 * 7)
        assert not f[inside].eq(7).any()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_on_views_that_begin_at_any_sixteen_bytes(bits):
    for dt, off in ((torch.bfloat16, 8), (torch.float32, 4)):
        t = group([700, 2048, 5001], dt, dt, bits, 31)
        for x in t:
            for name in ("param", "grad"):
                old = getattr(x, name)
                wide = torch.zeros(old.numel() + off, dtype=dt, device="cuda")
                wide[off:] = old
                setattr(x, name, wide[off:])
            assert x.param.data_ptr() % 32 == 16
        check_step(t, bits, H, 9, srq.SR, 5, 77)


def test_adamw_gradients_that_move_are_given_anew():
    t = group([300, 40], torch.float32, torch.float32, 32, 33)
    a = srq.AdamTensors(t)
    old = t[1].grad
    a.set_grad(1, torch.full((40,), 2.0, device="cuda"))
    old.fill_(math.nan)
    m = t[1].m.clone()
    s = status()
    srq.srq_adamw_step(a, **H, step=1, device_status=s)
    assert s.item() == 0 and torch.allclose(t[1].m, m * 0.9 + 0.2) and len(a) == 2
    with pytest.raises(ValueError, match="grad"):
        a.set_grad(1, torch.zeros(39, device="cuda"))


# --------------------------------------------------------------------------------------------
# streams and graphs
# --------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph_give_the_same_bits():
    g = gen(11)
    t, v, d = 3000, 700, 72
    ids, dout, table = make_ids("few", t, v, g, torch.int64), randn(g, t, d), randn(g, v, d)
    x, targets = make_logits(g, 90, 5003, torch.bfloat16, 0)
    old, adv, w = randn(g, 90, std=0.1) - 9, randn(g, 90), torch.full((90,), 1 / 90, device="cuda")
    off = torch.tensor([0, 20, 45, 60, 90], device="cuda")
    ws, ws2 = srq.new_workspace(srq.srq_embedding_workspace_bytes(t, v, d)), srq.new_workspace(srq.srq_preference_workspace_bytes(90))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def fresh():
        return dict(out=torch.empty((t, d), device="cuda"), dtable=torch.empty((v, d), device="cuda"), row=torch.empty(90, device="cuda"), loss=torch.empty(1, device="cuda"),
                    dx=torch.empty_like(x), pair=torch.empty(2, device="cuda"), logp=torch.empty(90, device="cuda"), dy=torch.empty_like(x),
                    adam=group([3000, 17], torch.bfloat16, torch.float32, 8, 12))

    def work(o, a):
        srq.srq_embedding_fwd(table, ids, o["out"], 3.0)
        srq.srq_embedding_bwd(dout, ids, o["dtable"], 3.0, ws=ws)
        srq.srq_policy_loss(x, targets, old, adv, w, None, o["row"], o["loss"], None, o["dx"])
        srq.srq_preference_loss(x, targets, old, off, o["pair"], None, o["logp"], o["dy"], ws=ws2)
        step.add_(1)
        srq.srq_adamw_step(a, **H, step_device=step, seed=4)

    def results(o):
        return [o[n] for n in ("out", "dtable", "row", "loss", "dx", "pair", "logp", "dy")] + [q for t in o["adam"] for q in (t.param, t.m, t.v, t.m_step, t.v_step)]
    first = fresh()
    a = srq.AdamTensors(first["adam"])
    for _ in range(3):
        work(first, a)
    torch.cuda.synchronize()
    second, side = fresh(), torch.cuda.Stream()
    a = srq.AdamTensors(second["adam"])
    step.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            work(second, a)
    torch.cuda.synchronize()
    third = fresh()
    a = srq.AdamTensors(third["adam"])
    step.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(third, a)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for p, q, r in zip(results(first), results(second), results(third)):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_launches_are_counted_and_nothing_is_allocated():
    g = gen(13)
    x, targets = make_logits(g, 50, 3000, torch.bfloat16, 0)
    z = randn(g, 50)
    dx, row, loss = torch.empty_like(x), torch.empty(50, device="cuda"), torch.empty(1, device="cuda")
    torch.cuda.synchronize()
    held, n = torch.cuda.memory_allocated(), srq.launch_count()
    srq.srq_policy_loss(x, targets, z - 9, z, z, None, row, loss, None, dx)
    assert srq.launch_count() == n + 2 and torch.cuda.memory_allocated() == held
