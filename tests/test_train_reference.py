"""CPU: the plain implementations that the GPU tests of the embedding, the losses and the AdamW step compare with, against
independent facts (differences, exact rationals, sums over all thresholds), and the host-side refusals of the entry points."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
import _train as ref
from paper_2511_00874_b200 import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = binding.OK, binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
P = 1 << 20                      # an "aligned pointer": the calls below must return before it is used


@pytest.fixture(scope="module")
def L():
    entry.build()
    return binding.lib()


# --------------------------------------------------------------------------------------------
# reference
# --------------------------------------------------------------------------------------------
def test_embedding_gradient_against_differences():
    ids = torch.tensor([2, 0, -1, 2, 4, 9, 2])
    table, dout = torch.randn(5, 3, dtype=torch.float64), torch.randn(7, 3, dtype=torch.float64)
    ok = (ids >= 0) & (ids < 5)
    f = lambda t: float((torch.where(ok[:, None], 1.5 * t[ids.clamp(0, 4)], 0.0) * dout).sum())  # noqa: E731
    got, _ = ref.embed_bwd(dout, ids, 5, 1.5)
    for i in range(5):
        for j in range(3):
            e = torch.zeros_like(table)
            e[i, j] = 1e-4
            assert abs((f(table + e) - f(table - e)) / 2e-4 - float(got[i, j])) < 1e-8


@pytest.mark.parametrize("with_ref", [False, True])
def test_policy_gradient_against_differences(with_ref):
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, targets = r(6, 9), torch.tensor([0, 8, 3, -1, 4, 2])
    old, adv, w = -2.2 + 0.3 * r(6), r(6), torch.tensor([0.2, 0.0, 0.3, 0.1, 0.2, 0.2], dtype=torch.float64)
    other = -2.2 + 0.3 * r(6) if with_ref else None

    def f(x):
        logp, _, p, _, _, counts = ref.logprob(x, targets, 0.7)
        loss, c = ref.policy(logp, old, adv, w * counts, other, 0.2, 0.3, 0.5)
        return float(loss.sum()), ref.dlogits(p, p * 0, targets, counts, c, c * 0, 0.7)[0]
    d = f(x)[1]
    assert not d[3].any() and not d[1].any()
    for i in range(6):
        for j in range(9):
            e = torch.zeros_like(x)
            e[i, j] = 1e-5
            assert abs((f(x + e)[0] - f(x - e)[0]) / 2e-5 - float(d[i, j])) < 1e-8


def test_preference_gradient_against_differences():
    g = torch.Generator().manual_seed(1)
    x, targets = torch.randn(8, 5, generator=g, dtype=torch.float64), torch.tensor([0, 1, -1, 3, 4, 0, 2, 2])
    other, offsets = torch.randn(8, generator=g, dtype=torch.float64), torch.tensor([1, 3, 4, 4, 7])

    def f(x):
        logp, _, p, _, _, counts = ref.logprob(x, targets)
        pair, _, c = ref.preference(torch.where(counts, logp - other, 0.0), offsets, 0.7, 0.1)
        return float(pair.mean()), ref.dlogits(p, p * 0, targets, counts, c, c * 0)[0]
    d = f(x)[1]
    for i in range(8):
        for j in range(5):
            e = torch.zeros_like(x)
            e[i, j] = 1e-5
            assert abs((f(x + e)[0] - f(x - e)[0]) / 2e-5 - float(d[i, j])) < 1e-9


@pytest.mark.parametrize("mantissa,top", [(3, 448.0), (4, 496.0)])
def test_codes_are_the_grid_and_rounding_has_no_bias(mantissa, top):
    values = ref.grid_value(np.arange(256 if mantissa == 4 else 127), mantissa)
    assert values[-1] == top and (np.diff(values) > 0).all()
    if mantissa == 3:
        want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
        assert np.array_equal(values, want)
    # the block's maximum is `top`, so the step is 1: the mean over all thresholds is the number itself, to half a threshold's step
    u = np.arange(65536)
    for x in (300.7, 1.0, 0.3, 0.017, 0.013, 2.0 ** -9, 2.0 ** -9 * 0.3):
        x = np.float32(x)
        got = []
        for a in range(0, 65536, 127):
            part = np.full(min(127, 65536 - a) + 1, x, dtype=np.float32)
            part[0] = top
            assert ref.block_steps(np.float32(top), top) == (1, 1)
            code, step = ref.encode(part, np.concatenate([[0], u[a:a + 127]]), top, mantissa)
            assert step[0] == 1 and code[0] == len(values) - 1
            got.append(ref.grid_value(code[1:], mantissa))
        got = np.concatenate(got)
        spacing = max(2.0 ** (np.floor(np.log2(x)) - mantissa), 2.0 ** (-6 - mantissa))
        assert abs(got.mean() - float(x)) <= spacing * 2.0 ** -17 * 1.01 and len(np.unique(got)) <= 2


def test_bf16_cut_has_the_mean_of_the_number():
    for x in (0.1, -3.3, 1.0):
        got = ref.cut_bf16(np.full(65536, x, dtype=np.float32), np.arange(65536))
        v, n = np.unique(got, return_counts=True)
        assert sum(Fraction(float(a)) * int(b) for a, b in zip(v, n)) == Fraction(float(np.float32(x))) * 65536


def test_step_sizes_of_second_moments():
    for m in (2.0 ** -120, 31 * 2.0 ** -124, np.nextafter(np.float32(31 * 2.0 ** -124), np.float32(1)), 1.0, 3e38):
        step, inv = ref.block_steps(np.float32(m), 496.0)
        exact = Fraction(496) / Fraction(float(np.float32(m)))
        if float(np.float32(m)) <= 31 * 2.0 ** -124:
            assert inv == 0 and step == 0
        else:
            assert Fraction(float(inv)) <= exact < Fraction(float(np.nextafter(inv, np.float32(np.inf)))) or not np.isfinite(np.nextafter(inv, np.float32(np.inf)))


def test_second_moments_keep_their_mean_under_repeated_rounding():
    # 4000 steps of a constant squared gradient: the coded moment settles at it.  The rounding's noise, 1.8 % of the moment a step,
    # is remembered for 1 / (1 - beta2) steps: a deviation of 5.8 % for one element at 0.95, 0.5 % for the mean of 127 over time.
    rng = np.random.default_rng(0)
    beta2 = 0.95
    g2 = (0.2 + rng.random(128)).astype(np.float32)
    v, mean = np.zeros(128, np.float32), np.zeros(128)
    for t in range(1200):
        v = (v * np.float32(beta2) + g2 * np.float32(1 - beta2)).astype(np.float32)
        code, step = ref.encode(v, rng.integers(0, 65536, 128), 496.0, 4)
        v = (ref.grid_value(code, 4).astype(np.float32) * step[0]).astype(np.float32)
        if t >= 200:
            mean += v / 1000
    # mean over 1000 steps of one element: 5.8 % * sqrt(2 / (0.05 * 1000)) = 1.2 %; four standard deviations
    assert np.abs(mean / g2 - 1).max() < 0.05 and abs((mean / g2).mean() - 1) < 0.004


# --------------------------------------------------------------------------------------------
# refusals
# --------------------------------------------------------------------------------------------
def test_embedding_refusals(L):
    def f(table=P, dt=0, rows=8, cols=24, ld=24, ids=P, it=1, t=5, out=P, odt=1, ldo=24, s=None):
        return int(L.srq_embedding_fwd(table, dt, rows, cols, ld, ids, it, t, 1.0, out, odt, ldo, s, None))
    for bad in (dict(table=None), dict(ids=None), dict(out=None), dict(dt=2), dict(odt=-1), dict(it=2), dict(rows=-1), dict(cols=-1), dict(t=-1), dict(ld=23),
                dict(ldo=23), dict(table=P + 8), dict(out=P + 8), dict(ids=P + 4), dict(s=P + 2)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(rows=1 << 31), dict(t=1 << 31), dict(cols=(1 << 20) + 1, ld=1 << 24, ldo=1 << 24)):
        assert f(**bad) == UNSUPPORTED, bad
    assert f(t=0, ids=None, out=None) == OK and f(cols=0, table=None, out=None) == OK

    need = int(L.srq_embedding_workspace_bytes(5, 8, 24))
    assert need > 0 and L.srq_embedding_workspace_bytes(-1, 8, 24) == 0 and L.srq_embedding_workspace_bytes(5, 8, (1 << 20) + 1) == 0

    def b(dout=P, dt=0, t=5, cols=24, ld=24, ids=P, it=0, rows=8, out=P, odt=0, ldo=24, acc=0, ws=P, nb=need, s=None):
        return int(L.srq_embedding_bwd(dout, dt, t, cols, ld, ids, it, rows, 1.0, out, odt, ldo, acc, ws, nb, s, None))
    for bad in (dict(dout=None), dict(ids=None), dict(out=None), dict(dt=2), dict(odt=2), dict(it=-1), dict(rows=-1), dict(cols=-1), dict(t=-1), dict(ld=23),
                dict(ldo=23), dict(acc=2), dict(dout=P + 8), dict(out=P + 8), dict(ids=P + 2), dict(ws=None), dict(ws=P + 128), dict(s=P + 1)):
        assert b(**bad) == INVALID, bad
    assert b(acc=1, odt=1) == UNSUPPORTED and b(t=1 << 31, nb=1 << 60) == UNSUPPORTED
    assert b(nb=need - 1) == WORKSPACE
    assert b(rows=0, out=None) == OK and b(cols=0, dout=None, out=None) == OK and b(t=0, dout=None, ids=None, acc=1) == OK


def bad_logits():
    return (dict(x=None), dict(t=None), dict(dt=3), dict(it=2), dict(rows=-1), dict(c=-1), dict(ld=39), dict(x=P + 8), dict(t=P + 4), dict(temp=0.0),
            dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")), dict(temp=1e-31), dict(temp=2e30), dict(s=P + 1))


def test_logprob_refusals(L):
    def f(x=P, dt=1, rows=4, c=40, ld=40, t=P, it=1, temp=1.0, logp=P, lse=None, s=None):
        return int(L.srq_logprob_fwd(x, dt, rows, c, ld, t, it, temp, logp, lse, s, None))
    for bad in bad_logits() + (dict(logp=None), dict(logp=P + 2), dict(lse=P + 2)):
        assert f(**bad) == INVALID, bad
    assert f(c=1 << 31, ld=1 << 31) == UNSUPPORTED
    assert f(rows=0, x=None, t=None, logp=None) == OK

    def b(x=P, dt=1, rows=4, c=40, ld=40, t=P, it=1, temp=1.0, lse=P, d=P, dx=P, ldx=40, s=None):
        return int(L.srq_logprob_bwd(x, dt, rows, c, ld, t, it, temp, lse, d, dx, ldx, s, None))
    for bad in bad_logits() + (dict(lse=None), dict(d=None), dict(dx=None), dict(dx=P + 8), dict(ldx=39), dict(ldx=48), dict(lse=P + 1), dict(d=P + 2)):
        assert b(**bad) == INVALID, bad                                    # (dx is x: the same pitch)
    assert b(rows=0, x=None, t=None, lse=None, d=None, dx=None) == OK and b(c=0, x=None, dx=None, ld=0, ldx=0) == OK


def test_policy_refusals(L):
    def f(x=P, dt=1, rows=4, c=40, ld=40, t=P, it=1, old=P, adv=P, w=P, r=None, temp=1.0, lo=0.2, hi=0.2, kl=0.0, rl=P, loss=P, logp=None, dx=2 * P, ldx=40, s=None, h=True):
        h = ctypes.byref(binding._Policy(temp, lo, hi, kl)) if h else None
        return int(L.srq_policy_loss(x, dt, rows, c, ld, t, it, old, adv, w, r, h, rl, loss, logp, dx, ldx, s, None))
    nan = float("nan")
    for bad in bad_logits() + (dict(h=None), dict(lo=-0.1), dict(hi=-0.1), dict(kl=-1.0), dict(lo=nan), dict(hi=nan), dict(kl=nan), dict(kl=float("inf")), dict(old=None),
                               dict(adv=None), dict(w=None), dict(rl=None), dict(rl=None, loss=None, dx=None), dict(old=P + 1), dict(adv=P + 1), dict(w=P + 2), dict(r=P + 2),
                               dict(rl=P + 1), dict(loss=P + 2), dict(logp=P + 2), dict(dx=P, ldx=48), dict(dx=P + 8), dict(ldx=39)):
        assert f(**bad) == INVALID, bad
    assert f(rows=0, loss=None, x=None, t=None, old=None, adv=None, w=None, rl=None, dx=None) == OK


def test_preference_refusals(L):
    need = int(L.srq_preference_workspace_bytes(4))
    assert need > 0 and L.srq_preference_workspace_bytes(-1) == 0

    def f(x=P, dt=1, rows=4, c=40, ld=40, t=P, it=1, r=P, o=P, ot=1, n=2, temp=1.0, beta=0.1, eps=0.0, pl=P, loss=P, logp=P, dx=2 * P, ldx=40, ws=P, nb=need, s=None, h=True):
        h = ctypes.byref(binding._Preference(temp, beta, eps)) if h else None
        return int(L.srq_preference_loss(x, dt, rows, c, ld, t, it, r, o, ot, n, h, pl, loss, logp, dx, ldx, ws, nb, s, None))
    for bad in bad_logits() + (dict(h=None), dict(beta=float("inf")), dict(eps=-0.1), dict(eps=1.1), dict(eps=float("nan")), dict(n=-1), dict(ot=2), dict(r=None), dict(o=None),
                               dict(pl=None), dict(logp=None), dict(o=P + 4), dict(r=P + 1), dict(pl=P + 1), dict(loss=P + 1), dict(logp=P + 1), dict(dx=P, ldx=48),
                               dict(ws=None), dict(ws=P + 64)):
        assert f(**bad) == INVALID, bad
    assert f(nb=need - 1) == WORKSPACE and f(n=1 << 31) == UNSUPPORTED
    assert f(n=0, loss=None, o=None, pl=None) == OK


def adam(**kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1, round=binding.SR, seed=0, tensor_id=0, lr_device=None, step_device=None, grad_scale=None)
    return ctypes.byref(binding._AdamW(*{**d, **kw}.values()))


def test_adamw_refusals(L):
    def f(h=None, bits=32, pdt=0, gdt=0, n=1, s=None, tensors=True, **t):
        e = (binding._AdamTensor * 1)(binding._AdamTensor(*{**dict(param=P, grad=P, m=P, v=P, m_step=P, v_step=P, n=4), **t}.values()))
        return int(L.srq_adamw_step(e if tensors else None, n, pdt, gdt, bits, h or adam(), s, None))
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=P + 8), dict(grad=P + 8), dict(m=P + 8), dict(v=P + 8)):
        assert f(n=1, **bad) == INVALID and f(bits=8, **bad) == INVALID, bad
    for bad in (dict(m_step=None), dict(v_step=None), dict(m_step=P + 2), dict(v_step=P + 2)):
        assert f(bits=8, **bad) == INVALID, bad
    e = (binding._AdamTensor * 1)(binding._AdamTensor(P, P, P, P, None, None, -1))
    assert int(L.srq_adamw_step(e, 1, 0, 0, 32, adam(), None, None)) == INVALID
    assert f(pdt=2) == INVALID and f(gdt=2) == INVALID and f(s=P + 1) == INVALID and f(tensors=False) == INVALID and f(n=-1) == INVALID
    assert f(bits=16) == UNSUPPORTED
    nan, inf = float("nan"), float("inf")
    for bad in (dict(lr=nan), dict(lr=inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-39),
                dict(eps=inf), dict(weight_decay=nan), dict(step=0), dict(round=7), dict(lr_device=P + 2), dict(step_device=P + 4), dict(grad_scale=P + 1)):
        assert f(h=adam(**bad)) == INVALID, bad
    for r in (binding.RTN, binding.SR8):
        assert f(h=adam(round=r)) == UNSUPPORTED
    assert f(n=0) == OK
    none = (binding._AdamTensor * 2)(binding._AdamTensor(None, None, None, None, None, None, 0), binding._AdamTensor(None, None, None, None, None, None, 0))
    assert int(L.srq_adamw_step(none, 2, 0, 0, 8, adam(), None, None)) == OK


def test_binding_refuses_what_is_not_on_the_device_or_has_another_shape():
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        binding.srq_embedding_fwd(x, ids, x)
    with pytest.raises(TypeError, match="int32 or int64"):
        binding.srq_embedding_bwd(x, ids.float(), x)
    with pytest.raises(ValueError, match="CUDA"):
        binding.srq_logprob_fwd(x, ids, torch.zeros(4))
    with pytest.raises(ValueError, match="on the device"):
        binding.AdamTensors([binding.AdamTensor(x, x, x, x)])
    with pytest.raises(ValueError, match="8 or 32"):
        binding.new_adam_state(x, 16)
