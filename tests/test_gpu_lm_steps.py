"""GPU: what lm.TokenModel does with steps that are refused, with rows that belong to no answer and with what its parts report, and its
gradients under the policy loss."""
import math

import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import binding, lm

pytestmark = pytest.mark.gpu
T, V, K, F = 130, 300, 256, 384


def model(layers=1, **kw):
    m = lm.TokenModel(T, V, K, F, layers, embedding_scale=50.0, seed=3, **kw)
    m.initialise(0.03)
    m.lr.fill_(1e-3)
    return m


def batch(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pick = lambda: torch.randint(0, V, (T,), generator=g, device="cuda")  # noqa: E731
    return pick(), pick(), torch.full((T,), 1.0 / T, device="cuda")


def state(m):
    out = [m.table, m.head, *m.norms] + [w for layer in m.layers for w in layer] + [m.step]
    for group in (m.decaying, m.plain):
        out += [x for t in group.tensors for x in (t.m, t.v, t.m_step, t.v_step) if x is not None]
    return out


def step(m, args, grad_scale=None):
    ids, targets, weight = args
    m.forward(ids)
    m.supervised(targets, weight)
    m.backward(ids, srq.block_sr(5, 10))
    m.update(grad_scale=grad_scale)


@pytest.mark.parametrize("state_bits", [8, 32])
@pytest.mark.parametrize("what", ["grad_scale", "lr"])
def test_a_refused_update_is_not_counted(what, state_bits):
    args, one = batch(), torch.ones(1, device="cuda")
    plain, other = model(state_bits=state_bits), model(state_bits=state_bits)
    for bad in (math.nan, math.inf, -math.inf):
        before = [x.clone() for x in state(other)]
        if what == "lr":
            other.lr.fill_(bad)
            step(other, args)
            other.lr.fill_(1e-3)
        else:
            step(other, args, torch.tensor([bad], device="cuda"))
        assert other.status.item() == binding.ERR_NONFINITE
        for a, b in zip(state(other), before):
            assert torch.equal(a, b)
        other.status.zero_()
        step(plain, args, one)
        step(other, args, one)
        assert other.status.item() == 0
        for a, b in zip(state(plain), state(other)):
            assert torch.equal(a, b)
    assert plain.step.item() == 3


def test_recorded_updates_count_themselves():
    args, scale = batch(1), torch.ones(1, device="cuda")
    eager, recorded = model(), model()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step(recorded, args, scale)
    for value in (math.nan, 0.5, math.inf, math.nan, 2.0, 1.0):
        scale.fill_(value)
        g.replay()
        if math.isfinite(value):
            step(eager, args, scale)
    torch.cuda.synchronize()
    assert recorded.step.item() == 3 and recorded.status.item() == binding.ERR_NONFINITE
    for a, b in zip(state(eager), state(recorded)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("where", ["gate", "up", "down", "gradient"])
def test_what_the_layers_report_reaches_the_model(where):
    # the last layer's codes hold a NaN: found while they are coded, before any product
    m = model(2)
    args = batch(2)
    step(m, args)
    assert m.status.item() == 0
    if where == "gradient":
        m.forward(args[0])
        m.supervised(*args[1:])
        m.dy.zero_()
        m.blocks[1].backward(torch.full((T, K), math.nan, dtype=torch.bfloat16, device="cuda"))
    else:
        m.layers[1][("gate", "up", "down").index(where)][5, 7] = math.nan
        m.load()
    assert m.status.item() == binding.ERR_NONFINITE


def test_policy_gradients_of_the_model_against_autograd():
    # ratios far from the clip's bounds (log 0.7 = -0.36, log 1.3 = 0.26), half of them inside: log ratios of +-0.02 and +-1.2.  The coded
    # logits have a deviation of 12 % of 0.5, so that none of the rows crosses over.
    import test_gpu_lm as path
    m = path.model()
    ids, targets, weight, _, _, adv = path.inputs(3)
    counts = (targets >= 0).double()
    gap = torch.tensor([0.02, 1.2, -0.02, -1.2], device="cuda").repeat(path.T // 4).double()
    logits, _, _ = path.reference(m, ids, lambda z: z.sum())
    assert logits.abs().max() < 4 and logits.std() < 0.6
    base = path.token_logp(logits, targets)
    old, ref = (base - gap).float(), (base + 0.1).float()

    def plain(logits):
        logp = path.token_logp(logits, targets)
        rho, d = torch.exp(logp - old.double()), ref.double() - logp
        row = -torch.minimum(rho * adv, rho.clamp(0.7, 1.3) * adv) + 0.2 * (torch.expm1(d) - d)
        return (row * weight.double() * counts).sum()
    _, value, want = path.reference(m, ids, plain)
    m.forward(ids)
    got = m.policy(targets, old, adv, weight, ref, clip_low=0.3, clip_high=0.3, kl_coef=0.2)
    assert abs(got.item() - value) < path.LIMIT * max(1.0, abs(value))
    m.backward(ids)
    assert m.status.item() == 0
    for name, g in path.gradients(m).items():
        assert path.rel(g, want[name]) < path.LIMIT, name


def test_a_step_moves_the_rows_of_all_its_tokens():
    m = model(2)
    ids, targets, weight = batch(3)
    ids[:9], targets[-7:] = -1, -100
    start = m.table.clone()
    step(m, (ids, targets, weight))
    moved = (m.table != start).any(1)
    assert moved[ids[(ids >= 0) & (targets >= 0)]].all() and m.status.item() == 0


def test_supervised_rows_of_weight_zero_do_not_count():
    m, other = model(), model()
    ids, targets, weight = batch(4)
    weight[[5, 60, 129]] = 0.0
    m.forward(ids)
    m.logits[5], m.logits[60, targets[60]] = math.nan, -math.inf             # not read; minus infinity times zero would be NaN
    loss = m.supervised(targets, weight)
    other.forward(ids)
    want = other.supervised(torch.where(weight != 0, targets, -1), weight)
    assert m.status.item() == 0 and loss.isfinite().all() and torch.equal(loss, want)
    assert torch.equal(m.logits, other.logits) and not m.logits[[5, 60, 129]].any()


def test_supervised_weights_of_another_size_are_refused():
    m, args = model(), batch(5)
    m.forward(args[0])
    for bad in (args[2][:1], args[2][:-1], args[2][:, None]):
        with pytest.raises(ValueError, match="weight"):
            m.supervised(args[1], bad)
    assert m.supervised(args[1], args[2]).isfinite().all()                   # and leave the model as it was
