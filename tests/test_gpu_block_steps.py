"""GPU: stochastic rounding to block codes with the step's number read on the device: the thresholds are those of tensor_id + step * 2^32,
and a recorded call draws new ones at every replay."""
import pytest
import torch

import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import lm, mlp

pytestmark = pytest.mark.gpu
STEPS = [0, 1, 77, 2 ** 31 + 5, 2 ** 32 + 1]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(*blocks):
    return [t.clone() for b in blocks for t in (b.codes, b.scale)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def quantize(x):
    rows, cols = x.shape
    rm, tr = srq.new_blocks(rows, cols), srq.new_blocks(cols, rows)
    return lambda q: srq.srq_quantize_blocks(x, q, rm, tr), (rm, tr)


def tiles(x):
    rows, cols = x.shape
    rm, tr = srq.new_blocks(rows, cols, 128), srq.new_blocks(cols, rows, 128)
    return lambda q: srq.srq_quantize_blocks(x, q, rm, tr), (rm, tr)


def requantize(x):
    rows, cols = x.shape
    src, rm, tr = srq.new_blocks(rows, cols), srq.new_blocks(rows, cols), srq.new_blocks(cols, rows)
    srq.srq_quantize_blocks(x, srq.BLOCK_RNE, src)
    src.scale.mul_(0.77)
    return lambda q: srq.srq_quantize_blocks(src, q, rm, tr), (rm, tr)


def norm(x):
    rows, cols = x.shape
    y, w = srq.new_blocks(rows, cols), torch.ones(cols, device="cuda")
    return lambda q: srq.srq_rmsnorm_fwd(x, None, w, 1e-5, y, q=q), (y,)


def glu(x):
    rows, cols = x.shape
    gate, up = srq.new_blocks(rows, cols), srq.new_blocks(rows, cols)
    srq.srq_quantize_blocks(x, srq.BLOCK_RNE, gate)
    srq.srq_quantize_blocks(x * 0.5 + 0.1, srq.BLOCK_RNE, up)
    dg, du = srq.new_blocks(rows, cols), srq.new_blocks(rows, cols)
    dgt, dut, ht = (srq.new_blocks(cols, rows) for _ in range(3))
    return lambda q: srq.srq_glu_bwd(x, gate, up, srq.SILU, q, dg, du, dgt, dut, ht), (dg, du, dgt, dut, ht)


@pytest.mark.parametrize("op", [quantize, tiles, requantize, norm, glu])
@pytest.mark.parametrize("rows,cols,dtype", [(256, 384, torch.bfloat16), (77, 203, torch.float32), (1, 40, torch.bfloat16)])
def test_thresholds_of_a_step(op, rows, cols, dtype):
    x = torch.randn(rows, cols, generator=gen(1), device="cuda").to(dtype)
    f, out = op(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    seen = []
    for t in STEPS:
        f(srq.block_sr(5, 9 + 2 ** 32, 3 * cols + 1))                       # something else in between
        step.fill_(t)
        f(srq.block_sr(5, 9, 12, step=step))
        got = codes(*out)
        f(srq.block_sr(5, 9 + (t << 32), 12))
        assert same(got, codes(*out)), t
        seen.append(got)
    if rows * cols > 1000:                                                  # (in one of the layouts: coded numbers may have nothing to round in theirs)
        assert all(not same(a, b) for i, a in enumerate(seen[:4]) for b in seen[:i])
    step.fill_(3)                                                           # rounding to nearest has no thresholds
    f(srq.BLOCK_RNE)
    nearest = codes(*out)
    f(srq.QSpec(8, srq.PER_BLOCK, srq.RNE, 5, 9, format=srq.GRID_E4M3, step=step))
    assert same(nearest, codes(*out))


def test_a_recorded_quantization_draws_new_thresholds_at_every_replay():
    x = torch.randn(300, 520, generator=gen(2), device="cuda")
    f, out = quantize(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    q = srq.block_sr(3, 4, step=step)
    f(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.add_(1)
        f(q)
    mean, n, first = torch.zeros(300, 520, dtype=torch.float64, device="cuda"), 64, None
    for t in range(1, n + 1):
        g.replay()
        got = codes(*out)
        mean += out[0].dequantize().double() / n
        first = mean * n if first is None else first
        f(srq.block_sr(3, 4 + (t << 32)))
        assert same(got, codes(*out))
    # independent thresholds: the error of the mean of n is 1 / sqrt(n) = 1/8 of one rounding's (n - 1 repeated ones: 1)
    assert (mean - x.double()).norm() < 0.2 * (first - x.double()).norm()


def test_the_feed_forward_block_passes_the_step_on():
    T, K, F = 200, 256, 384
    r = lambda *s: torch.randn(*s, generator=gen(sum(s)), device="cuda").bfloat16()  # noqa: E731
    m = mlp.GatedMLP(T, K, F)
    m.load(1 + 0.1 * r(K), r(F, K) / 16, r(F, K) / 16, r(K, F) / 16)
    x, dout = r(T, K), r(T, K + 1)[:, 1:].contiguous()
    m.forward(x)
    step = torch.full((1,), 6, dtype=torch.int64, device="cuda")
    grads = lambda: [t.clone() for t in (m.dx, m.dwg, m.dwu, m.dwd, m.dw)]  # noqa: E731
    m.backward(dout, None, srq.block_sr(7, 100, step=step))
    got = grads()
    m.backward(dout, None, srq.block_sr(7, 100 + (6 << 32)))
    assert same(got, grads())
    m.backward(dout, None, srq.block_sr(7, 100))
    assert not same(got, grads())


@pytest.mark.parametrize("recorded", [False, True])
def test_a_model_rounds_its_gradients_anew_at_every_step(recorded):
    T, V, K, F = 130, 300, 256, 384
    m = lm.TokenModel(T, V, K, F, 1, embedding_scale=50.0, seed=3)
    m.initialise(0.03)                                                      # the learning rate is 0: the weights stay
    ids, targets = torch.randint(0, V, (T,), generator=gen(4), device="cuda"), torch.randint(0, V, (T,), generator=gen(5), device="cuda")
    weight, q = torch.full((T,), 1.0 / T, device="cuda"), srq.block_sr(5, 10)

    def step():
        m.forward(ids)
        m.supervised(targets, weight)
        m.backward(ids, q)
        m.update()
    start = m.head.clone()
    run = step
    if recorded:
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        run = g.replay
        m.step.zero_()
    seen = []
    for t in range(4):
        run()
        seen.append([m.dl.codes.clone(), m.blocks[0].dout.codes.clone(), m.blocks[0].dgu.codes.clone(), m.dtable.clone()])
        srq.srq_quantize_blocks(m.logits, srq.block_sr(5, 10 + (t << 32)), m.dl)
        assert torch.equal(seen[-1][0], m.dl.codes)
    torch.cuda.synchronize()
    assert torch.equal(m.head, start) and m.step.item() == 4 and m.status.item() == 0
    for i in range(4):
        for a, b in zip(seen[i], seen[i - 1]):
            assert not torch.equal(a, b)
