"""GPU: a training step built from the library's operators (lm.TokenModel), against torch's autograd in 64 bits.

A product of two coded operands carries 2.6 % sqrt(2) of its norm (test_gpu_mlp.py).  On its way to a gradient an error passes through
the coded operands of one layer's forward (6) and backward pass (10), the logits (2) and their gradient's products (3): 2.6 % sqrt(21) = 12 %,
where logits are small enough for the probabilities not to magnify them (|z| < 1 here).  The bounds leave a factor of 1.5."""
import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import lm

pytestmark = pytest.mark.gpu
T, V, K, F = 200, 300, 256, 384
LIMIT = 0.026 * 21 ** 0.5 * 1.5


def model(layers=1, **kw):
    m = lm.TokenModel(T, V, K, F, layers, embedding_scale=50.0, seed=3, **kw)
    m.initialise(0.03)
    m.lr.fill_(1e-3)
    return m


def inputs(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, V // 4, (T,), generator=g, device="cuda")
    ids[-5:] = -1
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    targets[:3] = -100
    r = lambda std: std * torch.randn(T, generator=g, device="cuda")  # noqa: E731
    return ids, targets, torch.full((T,), 1.0 / T, device="cuda"), r(0.1) - 5.7, r(0.1) - 5.7, r(1.0)


def reference(m, ids, dlogits_of):
    """Gradients of the loss by autograd from the weights as they are: (logits, {name: gradient})."""
    leaf = lambda w: w.double().requires_grad_()  # noqa: E731
    table, head, norms = leaf(m.table), leaf(m.head), [leaf(w) for w in m.norms]
    layers = [[leaf(w) for w in layer] for layer in m.layers]
    norm = lambda r, w: r * torch.rsqrt(r.square().mean(1, keepdim=True) + m.eps) * w  # noqa: E731
    x = torch.where(ids[:, None] >= 0, table[ids.clamp(min=0)] * m.scale, 0.0)
    r = torch.zeros_like(x)
    for w, (g, u, d) in zip(norms, layers):
        r = x + r
        y = norm(r, w)
        x = (torch.nn.functional.silu(y @ g.t()) * (y @ u.t())) @ d.t()
    logits = norm(x + r, norms[-1]) @ head.t()
    loss = dlogits_of(logits)
    loss.backward()
    grads = {"table": table.grad, "head": head.grad}
    for i, (w, layer) in enumerate(zip(norms, layers)):
        grads.update({f"norm {i}": w.grad, f"wg {i}": layer[0].grad, f"wu {i}": layer[1].grad, f"wd {i}": layer[2].grad})
    grads["norm"] = norms[-1].grad
    return logits.detach(), float(loss.detach()), grads


def gradients(m):
    out = {"table": m.dtable, "head": m.dhead, "norm": m.dnorm}
    for i, b in enumerate(m.blocks):
        out.update({f"norm {i}": b.dw, f"wg {i}": b.dwg, f"wu {i}": b.dwu, f"wd {i}": b.dwd})
    return out


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


def token_logp(logits, targets):
    return torch.log_softmax(logits, 1).gather(1, targets.clamp(min=0)[:, None])[:, 0]


@pytest.mark.parametrize("loss", ["supervised", "policy", "preference"])
def test_gradients_of_a_step_against_autograd(loss):
    m = model()
    ids, targets, weight, old, ref, adv = inputs()
    counts = (targets >= 0).double()
    offsets, pair = torch.tensor([0, 60, 100, 170, T], device="cuda"), torch.empty(2, device="cuda")

    def plain(logits):
        logp = token_logp(logits, targets)
        if loss == "supervised":
            return -(logp * weight.double() * counts).sum()
        if loss == "policy":
            rho, d = torch.exp(logp - old.double()), ref.double() - logp
            row = -torch.minimum(rho * adv, rho.clamp(0.7, 1.3) * adv) + 0.2 * (torch.expm1(d) - d)
            return (row * weight.double() * counts).sum()
        s = [((logp - ref.double()) * counts)[a:b].sum() for a, b in zip(offsets.tolist(), offsets.tolist()[1:])]
        return -sum(torch.nn.functional.logsigmoid(0.1 * (s[2 * i] - s[2 * i + 1])) for i in range(2)) / 2
    logits, value, want = reference(m, ids, plain)
    assert logits.abs().max() < 4
    got = m.forward(ids)
    assert rel(got, logits) < LIMIT
    if loss == "supervised":
        got = m.supervised(targets, weight)
    elif loss == "policy":
        got = m.policy(targets, old, adv, weight, ref, clip_low=0.3, clip_high=0.3, kl_coef=0.2)
    else:
        got = m.preference(targets, ref, offsets, pair, beta=0.1)
    assert abs(got.item() - value) < LIMIT * max(1.0, abs(value))
    m.backward(ids)
    assert m.status.item() == 0
    if loss == "policy":
        # ratios near a bound may be clipped on one side only: few rows, but whole ones.  The gradient's size is compared instead.
        for name, g in gradients(m).items():
            assert 0.5 < float(g.double().norm() / want[name].norm()) < 2.0, name
        return
    for name, g in gradients(m).items():
        assert rel(g, want[name]) < LIMIT, name


def step(m, args, kind, offsets=None, pair=None):
    ids, targets, weight, old, ref, adv = args
    m.forward(ids)
    if kind == "policy":
        m.policy(targets, old, adv, weight, ref, kl_coef=0.1)
    elif kind == "preference":
        m.preference(targets, ref, offsets, pair)
    else:
        m.supervised(targets, weight)
    m.backward(ids, srq.block_sr(5, 10))
    m.update()


@pytest.mark.parametrize("state_bits", [8, 32])
@pytest.mark.parametrize("kind", ["supervised", "policy", "preference"])
def test_steps_recorded_and_replayed_give_the_same_weights(kind, state_bits):
    args, offsets, pair = inputs(1), torch.tensor([0, 60, 100, 170, T], device="cuda"), torch.empty(2, device="cuda")
    eager, recorded = model(2, state_bits=state_bits), model(2, state_bits=state_bits)
    start = eager.table.clone()
    for _ in range(3):
        step(eager, args, kind, offsets, pair)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(recorded, args, kind, offsets, pair)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert eager.status.item() == 0 and recorded.status.item() == 0
    weights = lambda m: [m.table, m.head, *m.norms] + [w for layer in m.layers for w in layer]  # noqa: E731
    for a, b in zip(weights(eager), weights(recorded)):
        assert a.isfinite().all() and torch.equal(a, b)
    moved = (eager.table != start).any(1)
    assert moved[args[0][args[0] >= 0].unique()].any() and eager.step.item() == 3


def test_clipping_by_a_device_scalar_and_a_step_that_is_not_finite():
    m = model()
    args = inputs(2)
    before = m.head.clone()
    m.forward(args[0])
    m.supervised(args[1], args[2])
    m.backward(args[0])
    m.update(grad_scale=torch.tensor([float("nan")], device="cuda"))
    assert m.status.item() == srq.binding.ERR_NONFINITE and torch.equal(m.head, before)
