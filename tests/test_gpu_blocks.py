"""GPU: the block-scaled operators against plain 64-bit implementations (tests/_blocks.py), at the sizes,
strides and masks where they can go wrong.  The bounds are derived there from the number of roundings."""
import numpy as np
import pytest
import torch

import _blocks as ref
import paper_2511_00874_b200 as srq
from paper_2511_00874_b200 import binding, synth

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
BF16_HALF_ULP = 2.0 ** -8         # eight significant bits: half a unit in the last place is 2^-8 of the number at most


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def blocks(rows, cols, tile=1, extra=0, poison=True):
    """A block matrix with a wide pitch; padding and contents start as 0x77."""
    codes = torch.full((rows, -(-cols // 16) * 16 + extra), 0x77, dtype=torch.uint8, device="cuda")
    nb = -(-cols // 128)
    scale = torch.full((-(-rows // tile), -(-nb // 4) * 4 + extra // 4), -7.0, device="cuda")
    b = srq.Blocks(codes[:, :cols], scale[:, :nb], tile)
    b.all_codes, b.all_scale = codes, scale
    return b


def padding_is_untouched(b):
    r, c = b.codes.shape
    assert bool((b.all_codes[:, c:] == 0x77).all()) and bool((b.all_scale[:, b.scale.shape[1]:] == -7.0).all())


def coded(x, tile=1):
    """Block codes of x by the reference quantizer."""
    c, s = ref.quantize(x.float().cpu().numpy(), tile)
    b = blocks(*x.shape, tile)
    b.codes.copy_(torch.from_numpy(c))
    b.scale.copy_(torch.from_numpy(s))
    return b


def numbers(b):
    return ref.values(b.codes, b.scale, b.tile_rows)


def skewed(rows, cols, seed, dtype=torch.float32):
    x = synth.normal((rows, cols), 1.0, seed, torch.float32, "cuda")
    return (x * torch.exp(0.8 * synth.normal((1, cols), 1.0, seed + 100, torch.float32, "cuda"))).to(dtype)


# --------------------------------------------------------------------------------------------
# quantizer: bit for bit
# --------------------------------------------------------------------------------------------
def check_quantizer(src, x, q, tile_rm, tile_tr, extra=0):
    r, c = x.shape
    rm = blocks(r, c, tile_rm, extra) if tile_rm else None
    tr = blocks(c, r, tile_tr, extra) if tile_tr else None
    s = status()
    srq.srq_quantize_blocks(src, q, rm, tr, device_status=s)
    assert s.item() == 0
    th = ref.thresholds(q, r, c) if q.round == srq.SR else None
    xn = x.float().cpu().numpy()
    for b, v, t, tile, name in ((rm, xn, th, tile_rm, "rm"), (tr, xn.T.copy(), None if th is None else th.T, tile_tr, "tr")):
        if b is None:
            continue
        codes, step = ref.quantize(v, tile, t)
        assert np.array_equal(b.scale.cpu().numpy(), step), name
        bad = np.argwhere(b.codes.cpu().numpy() != codes)
        assert bad.size == 0, f"{name}: {len(bad)} codes differ, first at {bad[0]}"
        padding_is_untouched(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tiles", [(1, 1), (128, 128), (1, 128), (128, None), (None, 1), (1, None), (None, 128)])
@pytest.mark.parametrize("q", [srq.BLOCK_RNE, srq.block_sr(3, 5, 0)], ids=["rne", "sr"])
def test_quantizer_layouts(dtype, tiles, q):
    x = skewed(300, 392, 1, DTYPES[dtype])
    check_quantizer(x, x, q, *tiles)


@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (128, 1), (1, 4096), (4096, 1), (3, 129), (129, 3), (127, 127), (257, 385), (1000, 17)])
def test_quantizer_odd_extents(shape):
    for k, q in enumerate((srq.BLOCK_RNE, srq.block_sr(2 ** 40 + 3, 2 ** 35 + 1, 2 ** 33 + 2), srq.block_sr(1, 2, 3))):
        for dtype in (torch.float32, torch.bfloat16):
            x = skewed(*shape, 7 + k, dtype)
            check_quantizer(x, x, q, 1, 1, extra=16)
            check_quantizer(x, x, q, 128, 128)


@pytest.mark.parametrize("pad", [1, 3, 4, 8])
def test_quantizer_strided_source(pad):
    for dtype in (torch.float32, torch.bfloat16):
        x = skewed(200, 256 + pad, 3, dtype)[:, :256]
        check_quantizer(x, x, srq.BLOCK_RNE, 1, 1)


@pytest.mark.parametrize("tile", [1, 128])
def test_requantizing_a_coded_matrix(tile):
    for shape in ((300, 392), (1, 130), (130, 1), (129, 256)):
        b = coded(skewed(*shape, 11), tile)
        x = (b.codes.contiguous().view(torch.float8_e4m3fn).float()
             * b.scale.repeat_interleave(tile, 0)[:shape[0]].repeat_interleave(128, 1)[:, :shape[1]])
        for q in (srq.BLOCK_RNE, srq.block_sr(9, 4)):
            check_quantizer(b, x, q, 1, 1)
            check_quantizer(b, x, q, 128, 128)


def test_quantizer_zero_tiny_and_wide_blocks():
    x = skewed(140, 400, 5)
    x[5] = 0
    x[:, 9] = 0
    x[:, 128:256] = 0                       # whole blocks with nothing in them
    x[7, 256:384] = 1e-40                   # too small to scale: stands for zero
    x[8, 256:384] = 7.0 * 2.0 ** -122
    x[9, 256:384] = 3e38
    x[10, 256:384] *= 2.0 ** -14
    for q in (srq.BLOCK_RNE, srq.block_sr(1, 1)):
        check_quantizer(x, x, q, 1, 1)
        check_quantizer(x, x, q, 128, 128)


def test_step_sizes_of_a_million_maxima():
    # one value per block: step size and (through the codes of the block's other values) reciprocal of every mantissa class
    g = np.random.default_rng(5)
    n = 1 << 20
    bits = g.integers(0, 1 << 23, n, dtype=np.uint32) | (g.integers(1, 254, n, dtype=np.uint32) << 23)
    bits[:4096] = (127 << 23) + np.arange(4096, dtype=np.uint32)                  # mantissas next to a power of two
    bits[4096:8192] = (128 << 23) - 1 - np.arange(4096, dtype=np.uint32)
    bits[8192:12288] = np.arange(4096, dtype=np.uint32) + np.float32(7.0).view(np.uint32) - 2048       # and next to 448 / 2^k
    m = bits.view(np.float32)
    x = np.zeros((n // 64, 64, 128), np.float32)
    x[..., 0] = m.reshape(-1, 64)
    f = g.uniform(0.4, 1.0, (n // 64, 64, 3)).astype(np.float32)
    x[..., 1:4] = x[..., :1] * f
    x = x.reshape(n // 64, 64 * 128)
    codes, step = ref.quantize(x)
    b = srq.new_blocks(n // 64, 64 * 128)
    srq.srq_quantize_blocks(torch.from_numpy(x).cuda(), srq.BLOCK_RNE, b)
    assert np.array_equal(b.scale.cpu().numpy(), step)
    assert np.array_equal(b.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_quantizer_reports_values_that_are_not_finite(value):
    x = skewed(130, 130, 5)
    x[129, 3] = value
    for rm, tr in ((1, None), (None, 1), (128, None), (None, 128)):
        s = status()
        srq.srq_quantize_blocks(x, srq.BLOCK_RNE, blocks(130, 130, rm) if rm else None, blocks(130, 130, tr) if tr else None, device_status=s)
        assert s.item() == binding.ERR_NONFINITE
        srq.srq_quantize_blocks(x, srq.BLOCK_RNE, blocks(130, 130, rm) if rm else None, blocks(130, 130, tr) if tr else None)     # no word: no report
    s = torch.full((1,), 7, dtype=torch.int32, device="cuda")                # the first report stays
    srq.srq_quantize_blocks(x, srq.BLOCK_RNE, blocks(130, 130), device_status=s)
    assert s.item() == 7


def test_quantizer_offsets_past_32_bits():
    rows, cols = 40000, 65536               # 2.6e9 elements
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for i in range(0, rows, 4000):
        x[i:i + 4000] = torch.randn((4000, cols), generator=g, device="cuda").to(torch.bfloat16)
    rm, tr = srq.new_blocks(rows, cols), srq.new_blocks(cols, rows)
    srq.srq_quantize_blocks(x, srq.BLOCK_RNE, rm, tr)
    for r in (0, 32767, 33001, rows - 1):
        c, s = ref.quantize(x[r:r + 1].float().cpu().numpy())
        assert np.array_equal(rm.codes[r:r + 1].cpu().numpy(), c) and np.array_equal(rm.scale[r:r + 1].cpu().numpy(), s)
    for k in (0, 53687, 60000, cols - 1):
        c, s = ref.quantize(x[:, k:k + 1].float().t().contiguous().cpu().numpy())
        assert np.array_equal(tr.codes[k:k + 1].cpu().numpy(), c) and np.array_equal(tr.scale[k:k + 1].cpu().numpy(), s)


# --------------------------------------------------------------------------------------------
# product
# --------------------------------------------------------------------------------------------
def check_product(m, n, k, ta, tb, dtype, accumulate=False, ldo_extra=0, seed=0):
    a, b = coded(skewed(m, k, seed), ta), coded(skewed(n, k, seed + 50), tb)
    want, bound = ref.product(numbers(a), numbers(b))
    whole = torch.full((m, n + ldo_extra), 3.5, dtype=DTYPES[dtype], device="cuda")
    out = whole[:, :n]
    s = status()
    if accumulate:
        start = skewed(m, n, seed + 9)
        out.copy_(start)
        want, bound = want + start.double(), bound + 2 * ref.ULP * (want + start.double()).abs()
    srq.srq_gemm_blocks(a, b, out, accumulate=accumulate, device_status=s)
    assert s.item() == 0
    if dtype == "bf16":
        bound = bound * 1.01 + BF16_HALF_ULP * 1.01 * want.abs()
    bad = (out.double() - want).abs() > bound + 1e-37
    assert not bad.any(), f"{int(bad.sum())} results off, first at {bad.nonzero()[0].tolist()}: {out[bad][0]} for {want[bad][0]}"
    assert bool((whole[:, n:] == 3.5).all())
    first = out.clone()
    if not accumulate:
        srq.srq_gemm_blocks(a, b, out)
        assert torch.equal(first, out), "the same product twice"


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 64, 65, 100, 128, 129, 255, 256, 257, 500])
def test_product_rows(m):
    check_product(m, 400, 640, 1, 128, "bf16", seed=m)
    check_product(m, 400, 640, 1, 1, "f32", seed=m)


@pytest.mark.parametrize("n,k", [(1, 1), (1, 128), (7, 129), (127, 16), (128, 127), (129, 1000), (255, 2048), (256, 4100), (257, 384), (1000, 513), (2560, 64)])
@pytest.mark.parametrize("m", [3, 200])
def test_product_extents(m, n, k):
    for tb in (1, 128):
        check_product(m, n, k, 1, tb, "f32", seed=n + k)
        check_product(m, n, k, 1, tb, "bf16", seed=n + k, ldo_extra=3)


@pytest.mark.parametrize("m", [40, 300])
@pytest.mark.parametrize("ta,tb", [(1, 1), (1, 128), (128, 1), (128, 128)])
def test_product_step_size_shapes(m, ta, tb):
    check_product(m, 520, 1300, ta, tb, "f32")


@pytest.mark.parametrize("m", [5, 130, 600])
@pytest.mark.parametrize("n", [256, 515])
def test_product_accumulates(m, n):
    for tb in (1, 128):
        check_product(m, n, 700, 1, tb, "f32", accumulate=True)


@pytest.mark.parametrize("m", [8, 300])
def test_product_pitches(m):
    for extra in (1, 4, 8, 12):
        for dtype in ("f32", "bf16"):
            check_product(m, 264, 256, 1, 128, dtype, ldo_extra=extra)


@pytest.mark.parametrize("m", [9, 260])
def test_product_step_pitch_without_vector_loads(m):
    a, b = coded(skewed(m, 900, 1)), coded(skewed(300, 900, 2), 128)
    wide = torch.full((m, 9), -1.0, device="cuda")
    wide[:, 1:].copy_(a.scale)                                       # base 4 bytes past alignment, odd pitch
    a2 = srq.Blocks(a.codes, wide[:, 1:], 1)
    want, bound = ref.product(numbers(a), numbers(b))
    out = torch.empty((m, 300), device="cuda")
    srq.srq_gemm_blocks(a2, b, out)
    assert not ((out.double() - want).abs() > bound).any()


def test_product_of_zero_blocks_and_of_an_empty_contraction():
    a, b = coded(torch.zeros(20, 256, device="cuda")), coded(skewed(30, 256, 1))
    out = torch.full((20, 30), 5.0, device="cuda")
    srq.srq_gemm_blocks(a, b, out)
    assert not out.any()
    st = binding.lib().srq_gemm_blocks(binding.ctypes.byref(a.c()), binding.ctypes.byref(b.c()), 20, 30, 0, out.fill_(5.0).data_ptr(), 0, 30, 0, None, None)
    torch.cuda.synchronize()
    assert st == 0 and not out.any()


@pytest.mark.parametrize("m,n,k", [(600, 1000, 2048), (1100, 4000, 2600), (5000, 1028, 2304), (300, 260, 20480)])
def test_product_last_round_in_halves(m, n, k):
    # tiles of a partly filled last round are added up from two halves of the contraction; pitches wider than the result
    for tb in (1, 128):
        check_product(m, n, k, 1, tb, "f32", seed=m, ldo_extra=4)
        check_product(m, n, k, 1, tb, "f32", seed=m, accumulate=True)


@pytest.mark.parametrize("n", [1027, 1100])
def test_product_of_many_rows_without_aligned_rows(n):
    # too many tiles for the few-token kernel; rows that no block store can take
    for tb in (1, 128):
        check_product(4099, n, 700, 1, tb, "bf16", ldo_extra=3)
        check_product(4099, n, 700, 1, tb, "f32", ldo_extra=1)
        check_product(4099, n, 700, 1, tb, "f32", accumulate=True, ldo_extra=1)


def test_product_long_contraction_and_many_tiles():
    check_product(300, 300, 20000, 1, 1, "f32")
    check_product(4, 256, 40000, 1, 128, "f32")
    check_product(2100, 5000, 256, 1, 128, "f32")


# --------------------------------------------------------------------------------------------
# norm
# --------------------------------------------------------------------------------------------
def norm_inputs(rows, cols, dtype, wdtype, residual, seed, pad=0):
    mk = lambda s: skewed(rows, cols + pad, s, DTYPES[dtype])[:, :cols]  # noqa: E731
    w = (1 + 0.2 * synth.normal((cols,), 1.0, seed + 3, torch.float32, "cuda")).to(DTYPES[wdtype])
    return mk(seed), mk(seed + 1) if residual else None, w


def check_norm(rows, cols, dtype, wdtype="f32", residual=True, seed=0, pad=0, sr=False):
    x, res, w = norm_inputs(rows, cols, dtype, wdtype, residual, seed, pad)
    y = blocks(rows, cols)
    r_out = torch.full((rows, cols + pad), 9.0, dtype=x.dtype, device="cuda")[:, :cols]
    y_out = torch.full((rows, cols + pad), 9.0, dtype=x.dtype, device="cuda")[:, :cols]
    rstd = torch.empty(rows, device="cuda")
    s = status()
    srq.srq_rmsnorm_fwd(x, res, w, EPS, y, r_out, rstd, y_out, device_status=s)
    assert s.item() == 0
    r, want_rstd, want = ref.norm(x.double(), None if res is None else res.double(), w.double(), EPS)
    rel = (ref.depth(cols) + 12) * ref.ULP                       # of 1 / rms: half the sum's, and of y
    half = BF16_HALF_ULP if dtype == "bf16" else 0.0                 # rounding of an output to its type
    assert not ((rstd.double() - want_rstd).abs() > rel * want_rstd).any()
    assert not ((r_out.double() - r).abs() > (half * 1.01 + ref.ULP) * r.abs()).any()
    assert not ((y_out.double() - want).abs() > (half * 1.01 + rel) * want.abs()).any()
    ref.check_coded(y.codes, y.scale, want, rel * want.abs(), "y")
    padding_is_untouched(y)
    # the parts on their own give the same
    y2, y3 = blocks(rows, cols), torch.empty((rows, cols), dtype=x.dtype, device="cuda")
    srq.srq_rmsnorm_fwd(x, res, w, EPS, y2)
    srq.srq_rmsnorm_fwd(x, res, w, EPS, None, y_out=y3)
    assert torch.equal(y.codes, y2.codes) and torch.equal(y.scale, y2.scale) and torch.equal(y_out, y3)


@pytest.mark.parametrize("rows", [1, 2, 7, 600])
@pytest.mark.parametrize("cols", [1, 5, 8, 128, 130, 256, 1000, 1024, 2048, 4096])
def test_norm_extents(rows, cols):
    check_norm(rows, cols, "bf16", "bf16", seed=rows + cols)
    check_norm(rows, cols, "f32", "f32", residual=False, seed=rows + cols)


@pytest.mark.parametrize("cols", [8192, 16392, 32768, 32776, 40001])
def test_norm_long_rows(cols):
    check_norm(3, cols, "f32")
    check_norm(2, cols, "bf16", "f32", residual=False)


@pytest.mark.parametrize("cols", [8193, 8200, 12288, 12290, 16384])
def test_norm_many_long_rows(cols):
    # more rows than SMs, whole groups of eight columns and others
    check_norm(300, cols, "f32")
    check_norm(300, cols, "f32", residual=False)
    check_norm(300, cols, "bf16", "f32", residual=False)


@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("wdtype", ["f32", "bf16"])
def test_norm_strides_and_types(pad, wdtype):
    for dtype in ("f32", "bf16"):
        check_norm(33, 520, dtype, wdtype, pad=pad)


def test_norm_stochastic_rounding_uses_the_stream_of_the_flat_index():
    for rows, cols, off in ((5, 640, 0), (4, 131, 2 ** 33 + 1)):
        x, res, w = norm_inputs(rows, cols, "f32", "f32", True, 3)
        y, y_out = blocks(rows, cols), torch.empty((rows, cols), device="cuda")
        q = srq.block_sr(11, 13, off)
        srq.srq_rmsnorm_fwd(x, res, w, EPS, y, y_out=y_out, q=q)
        codes, step = ref.quantize(y_out.cpu().numpy(), 1, ref.thresholds(q, rows, cols))
        assert np.array_equal(y.codes.cpu().numpy(), codes) and np.array_equal(y.scale.cpu().numpy(), step)


def test_norm_of_zero_rows_and_of_rows_that_are_not_finite():
    x = skewed(4, 512, 1)
    x[1] = 0
    y, rstd, s = blocks(4, 512), torch.empty(4, device="cuda"), status()
    srq.srq_rmsnorm_fwd(x, None, torch.ones(512, device="cuda"), EPS, y, rstd=rstd, device_status=s)
    assert s.item() == 0 and not (y.codes[1] & 0x7F).any() and not y.scale[1].any()
    assert abs(rstd[1].item() - EPS ** -0.5) < 1e-4 * EPS ** -0.5
    x[2, 7] = float("nan")
    srq.srq_rmsnorm_fwd(x, None, torch.ones(512, device="cuda"), EPS, y, device_status=s)
    assert s.item() == binding.ERR_NONFINITE


@pytest.mark.parametrize("cols,sr", [(512, False), (4096, False), (131, False), (40001, False), (640, True)])
def test_norm_reports_rows_whose_mean_square_leaves_binary32(cols, sr):
    # every value is finite, their squares are not: 1 / rms is 0 then, and so are the row's codes, which must not pass unnoticed
    q, w = srq.block_sr(1, 2) if sr else srq.BLOCK_RNE, torch.ones(cols, device="cuda")
    for rows in (3, 400):
        for big, want in ((1e15, 0), (3e19, binding.ERR_NONFINITE)):
            x = skewed(rows, cols, 1)
            x[rows - 1] = big
            s = status()
            srq.srq_rmsnorm_fwd(x, None, w, EPS, blocks(rows, cols), device_status=s, q=q)
            assert s.item() == want
            s = status()
            srq.srq_rmsnorm_fwd(x, None, w, EPS, None, y_out=torch.empty_like(x), device_status=s)
            assert s.item() == want
            srq.srq_rmsnorm_fwd(x, None, w, EPS, blocks(rows, cols), q=q)                  # no word: no report


def check_norm_bwd(rows, cols, dtype, wdtype="f32", residual=True, seed=0, pad=0):
    r, dres, w = norm_inputs(rows, cols, dtype, wdtype, residual, seed, pad)
    dy = skewed(rows, cols + pad, seed + 5, DTYPES[dtype])[:, :cols]
    rstd = (1 / torch.sqrt(r.double().square().mean(1) + EPS)).float()
    dx = torch.full((rows, cols + pad), 9.0, dtype=r.dtype, device="cuda")[:, :cols]
    dw = torch.full((cols,), 9.0, device="cuda")
    srq.srq_rmsnorm_bwd(dy, r, w, rstd, dres, dx, dw)
    args = (dy.double(), r.double(), w.double(), rstd.double())
    want, want_w = ref.norm_bwd(*args, None if dres is None else dres.double())
    n, rs = args[1] * args[3][:, None], args[3][:, None]
    prod = (args[0] * args[2] * n).abs()
    err = rs * (8 * ref.ULP * (args[0] * args[2]).abs() + n.abs() * (ref.depth(cols) + 12) * ref.ULP * prod.mean(1, keepdim=True)) + 4 * ref.ULP * want.abs()
    if dtype == "bf16":
        err = err * 1.01 + BF16_HALF_ULP * 1.01 * want.abs()
    bad = (dx.double() - want).abs() > err + 1e-37
    assert not bad.any(), f"dx: {int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}"
    bad = (dw.double() - want_w).abs() > (-(-rows // min(rows, 256)) + 80) * ref.ULP * (args[0] * n).abs().sum(0)
    assert not bad.any(), f"dw: {int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}"
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    srq.srq_rmsnorm_bwd(dy, r, w, rstd, dres, dx2)
    srq.srq_rmsnorm_bwd(dy, r, w, rstd, dres, None, dw2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("rows", [1, 3, 31, 513, 1500])
@pytest.mark.parametrize("cols", [1, 9, 128, 300, 1024, 4096])
def test_norm_backward_extents(rows, cols):
    check_norm_bwd(rows, cols, "f32", seed=rows)
    check_norm_bwd(rows, cols, "bf16", "bf16", residual=False, seed=rows)


@pytest.mark.parametrize("cols", [8192, 16384, 16392, 33001])
def test_norm_backward_long_rows(cols):
    check_norm_bwd(20, cols, "f32")
    check_norm_bwd(3, cols, "bf16", "f32")


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_norm_backward_strides(pad):
    for dtype in ("f32", "bf16"):
        check_norm_bwd(40, 520, dtype, "bf16", pad=pad)


def test_norm_backward_refuses_workspaces_that_are_not_device_memory():
    x, w, rstd, dw = skewed(600, 256, 1), torch.ones(256, device="cuda"), torch.ones(600, device="cuda"), torch.empty(256, device="cuda")
    n = srq.srq_rmsnorm_workspace_bytes(600, 256)
    for ws in (torch.empty(n, dtype=torch.uint8), torch.empty(n, dtype=torch.uint8).pin_memory(),
               torch.empty((1, 256), dtype=torch.uint8, device="cuda").expand(n // 256, 256)):
        with pytest.raises(ValueError, match="ws"):
            srq.srq_rmsnorm_bwd(x, x, w, rstd, None, None, dw, ws)
    with pytest.raises(binding.SrqError, match="workspace"):
        srq.srq_rmsnorm_bwd(x, x, w, rstd, None, None, dw, srq.new_workspace(n - 4))
    srq.srq_rmsnorm_bwd(x, x, w, rstd, None, None, dw, srq.new_workspace(n))


# --------------------------------------------------------------------------------------------
# gated block
# --------------------------------------------------------------------------------------------
KINDS = {"silu": srq.SILU, "gelu": srq.GELU}


def check_glu(t, f, k, kind, tile_w=128, tile_x=1, out=None, checkpoint=True, seed=0):
    x = coded(synth.normal((t, k), 1.0, seed, torch.float32, "cuda"), tile_x)
    wg, wu = (coded(synth.normal((f, k), 2.0 * k ** -0.5, seed + i, torch.float32, "cuda"), tile_w) for i in (1, 2))
    h, gate, up = blocks(t, f), blocks(t, f), blocks(t, f)
    h_out = None if out is None else torch.full((t, f + 3), 4.0, dtype=DTYPES[out], device="cuda")[:, :f]
    s = status()
    srq.srq_glu_fwd(x, wg, wu, KINDS[kind], h, gate if checkpoint else None, up if checkpoint else None, h_out, device_status=s)
    assert s.item() == 0
    (g, eg), (u, eu), (hh, eh) = ref.glu(numbers(x), numbers(wg), numbers(wu), kind)
    ref.check_coded(h.codes, h.scale, hh, eh, "h")
    padding_is_untouched(h)
    if checkpoint:
        ref.check_coded(gate.codes, gate.scale, g, eg, "gate")
        ref.check_coded(up.codes, up.scale, u, eu, "up")
        padding_is_untouched(gate)
        padding_is_untouched(up)
    if out:
        e = eh * 1.01 + (BF16_HALF_ULP * 1.01 * hh.abs() if out == "bf16" else 0)
        assert not ((h_out.double() - hh).abs() > e).any()
        only = torch.empty((t, f), dtype=DTYPES[out], device="cuda")        # h itself on its own, other pitch
        srq.srq_glu_fwd(x, wg, wu, KINDS[kind], None, h_out=only)
        assert torch.equal(only, h_out)


@pytest.mark.parametrize("t", [1, 4, 16, 17, 64, 65, 128, 129, 300, 513])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_glu_tokens(t, kind):
    check_glu(t, 384, 512, kind, seed=t)


@pytest.mark.parametrize("t", [3, 200])
@pytest.mark.parametrize("f,k", [(1, 1), (16, 100), (100, 640), (128, 128), (130, 129), (1000, 2048)])
def test_glu_extents(t, f, k):
    check_glu(t, f, k, "silu", out="f32")
    check_glu(t, f, k, "gelu", tile_w=1, out="bf16", checkpoint=False)


@pytest.mark.parametrize("t", [70, 400])
def test_glu_step_size_shapes(t):
    for tw in (1, 128):
        for tx in (1, 128):
            check_glu(t, 260, 700, "silu", tw, tx)


def test_glu_many_tiles():
    check_glu(2100, 2600, 256, "silu", checkpoint=False)
    check_glu(2100, 2600, 256, "silu", tile_w=1)


@pytest.mark.parametrize("t,f,k", [(5, 384, 512), (60, 400, 256), (400, 400, 256), (2100, 2608, 256), (2100, 2601, 256)])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_glu_each_checkpoint_on_its_own(t, f, k, kind):
    # either checkpoint may be left out, and what is written does not depend on the other (few tokens and CTA pairs; codes
    # through block stores and, where f is no multiple of 16, straight from registers)
    x = coded(synth.normal((t, k), 1.0, 1, torch.float32, "cuda"))
    wg, wu = (coded(synth.normal((f, k), 2.0 * k ** -0.5, i, torch.float32, "cuda"), 128) for i in (2, 3))

    def run(names):
        out = {n: blocks(t, f) for n in names}
        srq.srq_glu_fwd(x, wg, wu, KINDS[kind], out.get("h"), out.get("gate"), out.get("up"), None if "h" in out else torch.empty((t, f), device="cuda"))
        for b in out.values():
            padding_is_untouched(b)
        return out
    both = run(("h", "gate", "up"))
    for names in (("h", "gate"), ("h", "up"), ("gate",), ("up",), ("gate", "up"), ("h",)):
        for n, b in run(names).items():
            assert torch.equal(b.codes, both[n].codes) and torch.equal(b.scale, both[n].scale), (names, n)


def test_glu_saturated_gates():
    # gates far out on both sides: the logistic function reaches 0 and 1
    t, f, k = 150, 256, 128
    x = coded(synth.normal((t, k), 1.0, 1, torch.float32, "cuda") * 100)
    wg = coded(synth.normal((f, k), 1.0, 2, torch.float32, "cuda"))
    for rows in (t, 20):
        xs = srq.Blocks(x.codes[:rows], x.scale[:rows], 1)
        for kind in KINDS:
            h, h_out = blocks(rows, f), torch.empty((rows, f), device="cuda")
            srq.srq_glu_fwd(xs, wg, wg, KINDS[kind], h, h_out=h_out)
            assert bool(torch.isfinite(h_out).all())
            (_, _), (_, _), (hh, eh) = ref.glu(numbers(xs), numbers(wg), numbers(wg), kind)
            assert not ((h_out.double() - hh).abs() > eh + 1e-30).any()


@pytest.mark.parametrize("t", [20, 300])
def test_glu_reports_values_that_are_not_finite(t):
    f, k = 300, 256
    x = coded(synth.normal((t, k), 1.0, 1, torch.float32, "cuda"))
    wg, wu = (coded(synth.normal((f, k), 1.0, i, torch.float32, "cuda"), 128) for i in (2, 3))
    bad_row = srq.Blocks(x.codes, x.scale.clone(), 1)
    bad_row.scale[t - 1, 1] = float("inf")
    bad_code = srq.Blocks(x.codes.clone(), x.scale, 1)
    bad_code.codes[3, 7] = 0x7F
    for src, want in ((x, 0), (bad_row, binding.ERR_NONFINITE), (bad_code, binding.ERR_NONFINITE)):
        for names in (("h",), ("gate",), ("up",), ("h", "gate", "up")):
            s = status()
            srq.srq_glu_fwd(src, wg, wu, srq.SILU, **{"h": None, **{n: blocks(t, f) for n in names}}, h_out=torch.empty((t, f), device="cuda"), device_status=s)
            assert s.item() == want, names
            srq.srq_glu_fwd(src, wg, wu, srq.GELU, **{"h": None, **{n: blocks(t, f) for n in names}}, h_out=torch.empty((t, f), device="cuda"))


def check_glu_bwd(t, f, dtype, kind, which=("dg", "du", "dg_t", "du_t", "h_t"), pad=0, seed=0):
    gate, up = coded(synth.normal((t, f), 1.5, seed, torch.float32, "cuda")), coded(skewed(t, f, seed + 1))
    dh = (1e-3 * skewed(t, f + pad, seed + 2)).to(DTYPES[dtype])[:, :f]
    out = {n: (blocks(f, t) if n.endswith("_t") else blocks(t, f)) for n in which}
    s = status()
    srq.srq_glu_bwd(dh, gate, up, KINDS[kind], srq.BLOCK_RNE, **out, device_status=s)
    assert s.item() == 0
    (dg, edg), (du, edu), (h, eh) = ref.glu_bwd(dh.double(), numbers(gate), numbers(up), kind)
    # g and u are formed as one binary32 product of code and step size
    edg, edu, eh = edg + 8 * ref.ULP * dg.abs(), edu + 8 * ref.ULP * du.abs(), eh + 8 * ref.ULP * h.abs()
    for n, b in out.items():
        v, e = {"dg": (dg, edg), "du": (du, edu), "h_": (h, eh)}[n[:2]]
        if n.endswith("_t"):
            v, e = v.t().contiguous(), e.t().contiguous()
        ref.check_coded(b.codes, b.scale, v, e, n)
        padding_is_untouched(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("t,f", [(1, 1), (1, 384), (2, 130), (128, 128), (129, 16), (300, 260), (513, 640)])
def test_glu_backward(dtype, kind, t, f):
    check_glu_bwd(t, f, dtype, kind, seed=t)


@pytest.mark.parametrize("which", [("dg",), ("du_t",), ("h_t",), ("dg", "du"), ("dg_t", "du_t"), ("du", "h_t")])
def test_glu_backward_any_subset(which):
    check_glu_bwd(200, 200, "bf16", "silu", which)


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_glu_backward_strided_gradient(pad):
    for dtype in ("f32", "bf16"):
        check_glu_bwd(150, 256, dtype, "gelu", pad=pad)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_glu_backward_saturated_gates(kind):
    # gates far out on both sides, up to where their squares leave binary32: the slope is 0 or 1 there, not infinity times 0
    t, f = 140, 260
    mag = torch.tensor([3.0, 50.0, 1e4, 1e12, 1.5e19, 2e19, 3e38], device="cuda")
    sign = torch.where(synth.normal((t, f), 1.0, 1, torch.float32, "cuda") > 0, 1.0, -1.0)
    gate = coded(sign * mag[torch.arange(t, device="cuda") % 7][:, None])
    up = coded(synth.normal((t, f), 1.0, 2, torch.float32, "cuda").clamp(-0.9, 0.9))
    dh = synth.normal((t, f), 1.0, 3, torch.float32, "cuda").clamp(-0.9, 0.9)
    out = {n: (blocks(f, t) if n.endswith("_t") else blocks(t, f)) for n in ("dg", "du", "dg_t", "du_t", "h_t")}
    s = status()
    srq.srq_glu_bwd(dh, gate, up, KINDS[kind], srq.BLOCK_RNE, **out, device_status=s)
    assert s.item() == 0
    (dg, edg), (du, edu), (h, eh) = ref.glu_bwd(dh.double(), numbers(gate), numbers(up), kind)
    for n, b in out.items():
        v, e = {"dg": (dg, edg), "du": (du, edu), "h_": (h, eh)}[n[:2]]
        e = e + 8 * ref.ULP * v.abs()
        if n.endswith("_t"):
            v, e = v.t().contiguous(), e.t().contiguous()
        ref.check_coded(b.codes, b.scale, v, e, n)


def test_glu_backward_stochastic_rounding_streams():
    t, f = 140, 264
    gate, up = coded(skewed(t, f, 1)), coded(skewed(t, f, 2))
    dh = skewed(t, f, 3)
    q = srq.block_sr(21, 40, 8)
    out = {n: (blocks(f, t) if n.endswith("_t") else blocks(t, f)) for n in ("dg", "du", "dg_t", "du_t", "h_t")}
    srq.srq_glu_bwd(dh, gate, up, srq.SILU, q, **out)
    near = {n: (blocks(f, t) if n.endswith("_t") else blocks(t, f)) for n in out}
    srq.srq_glu_bwd(dh, gate, up, srq.SILU, srq.BLOCK_RNE, **near)
    (dg, _), (du, _), (h, _) = ref.glu_bwd(dh.double(), numbers(gate), numbers(up), "silu")
    for n, b in out.items():
        assert torch.equal(b.scale, near[n].scale)
        v = {"dg": dg, "du": du, "h_": h}[n[:2]]
        spec = srq.block_sr(21, 40 + {"dg": 0, "du": 1, "h_": 2}[n[:2]], 8)
        th = torch.from_numpy(ref.thresholds(spec, t, f)).cuda().double() * 2.0 ** -24
        if n.endswith("_t"):
            v, th = v.t(), th.t()
        # rounded up exactly where the threshold lies under the fraction, wherever binary32 cannot have moved it across
        d = b.scale.double().repeat_interleave(128, 1)[:, :v.shape[1]]
        q_ = v / d
        sp = ref._spacing(q_)
        frac = q_ / sp - torch.floor(q_ / sp)
        got = b.codes.contiguous().view(torch.float8_e4m3fn).double()
        want = (torch.floor(q_ / sp) + (th < frac)) * sp
        clear = ((th - frac).abs() > 1e-3) & (frac > 1e-3) & (frac < 1 - 1e-3)
        assert bool((got == want)[clear].all()) and clear.double().mean() > 0.95


def test_gradients_of_a_concatenated_matrix():
    # dX = dg Wg + du Wu as one product over 2 F: both halves written next to each other through pitched views
    t, f, k = 200, 256, 300
    gate, up = coded(skewed(t, f, 1)), coded(skewed(t, f, 2))
    both = srq.new_blocks(t, 2 * f)
    half = lambda i: srq.Blocks(both.codes[:, i * f:(i + 1) * f], both.scale[:, i * f // 128:(i + 1) * f // 128], 1)  # noqa: E731
    srq.srq_glu_bwd(skewed(t, f, 3), gate, up, srq.SILU, srq.BLOCK_RNE, half(0), half(1))
    w = skewed(2 * f, k, 4)                                         # [Wg; Wu]
    w_t = srq.new_blocks(k, 2 * f, 128)
    srq.srq_quantize_blocks(w, srq.BLOCK_RNE, None, w_t)
    out = torch.empty((t, k), device="cuda")
    srq.srq_gemm_blocks(both, w_t, out)
    want, bound = ref.product(ref.values(both.codes, both.scale), ref.values(w_t.codes, w_t.scale, 128))
    assert not ((out.double() - want).abs() > bound).any()


# --------------------------------------------------------------------------------------------
# streams, capture, launches
# --------------------------------------------------------------------------------------------
def test_operators_run_on_the_current_stream_and_in_a_graph():
    t, f, k = 96, 256, 256
    x, w = skewed(t, k, 1, torch.bfloat16), torch.ones(k, device="cuda", dtype=torch.bfloat16)
    wg, wu = coded(synth.normal((f, k), 0.06, 2, torch.float32, "cuda"), 128), coded(synth.normal((f, k), 0.06, 3, torch.float32, "cuda"), 128)
    wd = coded(synth.normal((k, f), 0.06, 4, torch.float32, "cuda"), 128)
    y, h, out = srq.new_blocks(t, k), srq.new_blocks(t, f), torch.empty((t, k), dtype=torch.bfloat16, device="cuda")

    def step():
        srq.srq_rmsnorm_fwd(x, None, w, EPS, y)
        srq.srq_glu_fwd(y, wg, wu, srq.SILU, h)
        srq.srq_gemm_blocks(h, wd, out)

    n0 = srq.launch_count()
    step()
    assert srq.launch_count() - n0 == 3
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    x.mul_(-1)                                                      # the graph reads its inputs anew
    g.replay()
    torch.cuda.synchronize()
    replayed = out.clone()
    step()
    torch.cuda.synchronize()
    assert torch.equal(out, replayed)


# --------------------------------------------------------------------------------------------
# nothing to do: torch gives a null pointer for a tensor without elements
# --------------------------------------------------------------------------------------------
NONE = [(0, 200), (5, 0), (0, 0)]


@pytest.mark.parametrize("r,c", NONE)
def test_quantizer_without_elements(r, c):
    for x in (torch.empty((r, c), device="cuda"), torch.empty((r, c), dtype=torch.bfloat16, device="cuda"), srq.new_blocks(r, c), srq.new_blocks(r, c, 128)):
        for q in (srq.BLOCK_RNE, srq.block_sr(1, 2)):
            for tile in (1, 128):
                rm, tr = srq.new_blocks(r, c, tile), srq.new_blocks(c, r, tile)
                srq.srq_quantize_blocks(x, q, rm, tr, device_status=status())
                srq.srq_quantize_blocks(x, q, rm)
                srq.srq_quantize_blocks(x, q, None, tr)
    with pytest.raises(binding.SrqError):                            # a call that asks for nothing stays an error
        srq.srq_quantize_blocks(torch.empty((r, c), device="cuda"), srq.BLOCK_RNE)


@pytest.mark.parametrize("m,n,k", [(0, 200, 256), (200, 0, 256), (0, 0, 0), (0, 10, 0), (3, 200, 0), (300, 40, 0), (1, 1, 0)])
def test_product_without_elements(m, n, k):
    for tile in (1, 128):
        for dtype in (torch.float32, torch.bfloat16):
            whole = torch.full((m, n + 3), 5.0, dtype=dtype, device="cuda")
            out = whole[:, :n]
            srq.srq_gemm_blocks(srq.new_blocks(m, k), srq.new_blocks(n, k, tile), out, device_status=status())
            assert not out.any() and bool((whole[:, n:] == 5.0).all())               # an empty contraction is zero
    out = torch.full((m, n), 5.0, device="cuda")
    srq.srq_gemm_blocks(srq.new_blocks(m, k), srq.new_blocks(n, k), out, accumulate=True)
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("r,c", NONE)
def test_norm_without_elements(r, c):
    for dtype in (torch.float32, torch.bfloat16):
        e = lambda: torch.empty((r, c), dtype=dtype, device="cuda")  # noqa: E731
        w, rstd = torch.ones(c, dtype=dtype, device="cuda"), torch.empty(r, device="cuda")
        srq.srq_rmsnorm_fwd(e(), e(), w, EPS, srq.new_blocks(r, c), e(), rstd, e(), device_status=status())
        srq.srq_rmsnorm_fwd(e(), None, w, EPS, None, y_out=e())
        dw = torch.full((c,), 5.0, device="cuda")
        srq.srq_rmsnorm_bwd(e(), e(), w, rstd, e(), e(), dw)
        assert not dw.any()                                           # a sum over no rows
        srq.srq_rmsnorm_bwd(e(), e(), w, rstd, None, e())
        dw.fill_(5.0)
        srq.srq_rmsnorm_bwd(e(), e(), w, rstd, None, None, dw)
        assert not dw.any()


@pytest.mark.parametrize("t,f", NONE)
@pytest.mark.parametrize("act", [srq.SILU, srq.GELU])
def test_glu_without_elements(t, f, act):
    k = 256
    nb = srq.new_blocks
    h_out = torch.empty((t, f), device="cuda")
    for tile in (1, 128):
        srq.srq_glu_fwd(nb(t, k), nb(f, k, tile), nb(f, k, tile), act, nb(t, f), nb(t, f), nb(t, f), h_out, device_status=status())
        srq.srq_glu_fwd(nb(t, k), nb(f, k, tile), nb(f, k, tile), act, None, h_out=h_out)
    for dtype in (torch.float32, torch.bfloat16):
        dh = torch.empty((t, f), dtype=dtype, device="cuda")
        srq.srq_glu_bwd(dh, nb(t, f), nb(t, f), act, srq.BLOCK_RNE, nb(t, f), nb(t, f), nb(f, t), nb(f, t), nb(f, t), device_status=status())
