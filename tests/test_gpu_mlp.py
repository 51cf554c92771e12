"""GPU: the feed-forward block built from the block-scaled operators, against torch's autograd in 64 bits.

E4M3 rounds to within 2^-4 of a number, uniformly over its step: an rms of 2^-4 / sqrt(3) times the mean of (step /
largest step), about 2.6 %.  A product of two coded operands carries 2.6 % sqrt(2) of its norm, and the errors of a
chain add in squares: out 2.6 % sqrt(2 + 2 + 2) (norm and weights, h, down projection), the input gradient through
dout, Wd, the checkpoints, dg and du, and the weights about 2.6 % sqrt(10) = 8 %.  Stochastic rounding has sqrt(2) times
the rms of rounding to nearest on the gradients.  The bounds below leave a factor of 1.5."""
import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import mlp, synth

pytestmark = pytest.mark.gpu


def reference(x, res, w, wg, wu, wd, dout, dr, act, eps):
    leaves = [t.double().requires_grad_() for t in (x, w, wg, wu, wd)]
    xx, ww, g, u, d = leaves
    r = xx + res.double()
    y = r * torch.rsqrt(r.square().mean(1, keepdim=True) + eps) * ww
    f = torch.nn.functional.silu if act == srq.SILU else lambda t: torch.nn.functional.gelu(t, approximate="tanh")
    out = (f(y @ g.t()) * (y @ u.t())) @ d.t()
    ((out * dout.double()).sum() + (r * dr.double()).sum()).backward()
    return out.detach(), [t.grad for t in leaves]


@pytest.mark.parametrize("T,K,F,act,dtype,sr", [(300, 256, 384, srq.SILU, torch.bfloat16, False), (300, 256, 384, srq.GELU, torch.float32, True),
                                                (5, 384, 256, srq.SILU, torch.bfloat16, False), (1100, 520, 640, srq.GELU, torch.bfloat16, False)])
def test_mlp_forward_and_backward_against_autograd(T, K, F, act, dtype, sr):
    mk = lambda r, c, std, seed: synth.normal((r, c), std, seed, dtype, "cuda")  # noqa: E731
    x, res, dout, dr = mk(T, K, 1.0, 1), mk(T, K, 1.0, 2), mk(T, K, 1e-2, 3), mk(T, K, 1e-3, 4)
    w = (1 + 0.1 * synth.normal((K,), 1.0, 5, torch.float32, "cuda")).to(dtype)
    wg, wu, wd = mk(F, K, K ** -0.5, 6), mk(F, K, K ** -0.5, 7), mk(K, F, F ** -0.5, 8)
    m = mlp.GatedMLP(T, K, F, act, dtype)
    m.load(w, wg, wu, wd)
    out = m.forward(x, res)
    dx = m.backward(dout, dr, srq.block_sr(7, 100) if sr else srq.BLOCK_RNE)
    assert m.status.item() == 0
    want, grads = reference(x, res, w, wg, wu, wd, dout, dr, act, m.eps)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, want) < 0.026 * 6 ** 0.5 * 1.5
    limit = 0.026 * 10 ** 0.5 * 1.5 * (2 ** 0.5 if sr else 1.0)
    for name, got, ref in (("dx", dx, grads[0]), ("dw", m.dw, grads[1]), ("dwg", m.dwg, grads[2]), ("dwu", m.dwu, grads[3]), ("dwd", m.dwd, grads[4])):
        assert rel(got, ref) < limit, name
    # the same step again, recorded and replayed, gives the same bits
    first = [t.clone() for t in (out, dx, m.dw, m.dwg, m.dwu, m.dwd)]
    q = srq.block_sr(7, 100) if sr else srq.BLOCK_RNE
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.forward(x, res)
        m.backward(dout, dr, q)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, (m.out, m.dx, m.dw, m.dwg, m.dwu, m.dwd)):
        assert torch.equal(a, b)


def test_mlp_refuses_hidden_sizes_that_do_not_fill_blocks():
    with pytest.raises(ValueError, match="multiple of 128"):
        mlp.GatedMLP(4, 128, 200)


def test_mlp_of_no_tokens_has_zero_gradients():
    K, F = 256, 384
    m = mlp.GatedMLP(0, K, F)
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    wg, wu, wd = (synth.normal(s, 0.05, i, torch.bfloat16, "cuda") for i, s in enumerate([(F, K), (F, K), (K, F)]))
    m.load(w, wg, wu, wd)
    e = torch.empty((0, K), dtype=torch.bfloat16, device="cuda")
    assert m.forward(e, e).shape == (0, K) and m.backward(e, e).shape == (0, K)
    assert m.status.item() == 0
    for g in (m.dw, m.dwg, m.dwu, m.dwd):
        assert not g.any()


def test_mlp_rounds_each_weight_with_thresholds_of_its_own():
    K, F = 256, 256
    m = mlp.GatedMLP(4, K, F)
    one = synth.normal((F, K), 0.05, 1, torch.float32, "cuda")
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    m.load(w, one, one, one, srq.block_sr(3, 50))
    codes = [b.codes for b in (m.wg, m.wu, m.wd)]
    for i in range(3):
        want = srq.new_blocks(F, K, 128)
        srq.srq_quantize_blocks(one, srq.block_sr(3, 50 + i), want)
        assert torch.equal(codes[i], want.codes)
    for a, b in ((0, 1), (0, 2), (1, 2)):
        assert (codes[a] != codes[b]).double().mean() > 0.1           # the same numbers, rounded independently
    m.load(w, one, one, one)                                          # to nearest there is nothing to choose
    assert torch.equal(m.wg.codes, m.wu.codes) and torch.equal(m.wg.codes, m.wd.codes)
