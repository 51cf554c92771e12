"""CPU: the plain implementations the GPU tests compare with, against independent facts (gradients against
differences, the quantizer against the other quantizers' oracle), and the host-side refusals of the
block-scaled entry points."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
import oracle
from paper_2511_00874_b200 import binding
import _blocks as ref


@pytest.fixture(scope="module")
def L():
    entry.build()
    return binding.lib()


# --------------------------------------------------------------------------------------------
# reference
# --------------------------------------------------------------------------------------------
def test_step_sizes_and_sr_codes_agree_with_the_oracle_on_one_block():
    # one row of 128: a per-tensor E4M3 quantization point and a 1 x 128 block are the same thing
    entry.build()
    for seed in range(4):
        x = np.random.default_rng(seed).normal(size=(1, 128)).astype(np.float32) * np.float32(10.0 ** (3 * seed - 4))
        q = binding.block_sr(seed + 1, 7, 12)
        codes, step = ref.quantize(x, 1, ref.thresholds(q, 1, 128))
        o = oracle.sr_quantize_e4m3(x, oracle.QSpec(8, oracle.PER_TENSOR, oracle.SR, seed + 1, 7, 12), True, False)
        assert np.array_equal(codes, o[0]) and np.array_equal(step.ravel(), np.asarray(o[1]).ravel())


def test_rounding_is_to_nearest_and_a_tiny_block_is_zero():
    x = np.zeros((2, 128), np.float32)
    x[0, :4] = [448.0, 1.0625, 1.1875, -1.0625]       # ties between 1 and 1.125, 1.125 and 1.25
    codes, step = ref.quantize(x)
    v = ref.values(torch.from_numpy(codes), torch.from_numpy(step))
    assert v[0, :4].tolist() == [448.0, 1.0, 1.25, -1.0]
    x[1, 0] = 7.0 * 2.0 ** -122
    codes, step = ref.quantize(x)
    assert step[1, 0] == 0 and not codes[1].any()
    x[1, 0] = np.nextafter(np.float32(x[1, 0]), np.float32(1))
    assert ref.quantize(x)[1][1, 0] > 0


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_gradients_against_differences(kind):
    g = torch.linspace(-6, 6, 301, dtype=torch.float64)
    u = torch.cos(3 * g) + 0.3
    dh = torch.sin(g) + 1.5
    (dg, _), (du, _), (h, _) = ref.glu_bwd(dh, g, u, kind)
    e = 1e-5
    f = lambda gg, uu: (dh * ref.act(gg, kind)[0] * uu)  # noqa: E731
    assert torch.allclose(dg, (f(g + e, u) - f(g - e, u)) / (2 * e), rtol=1e-7, atol=1e-9)
    assert torch.allclose(du, (f(g, u + e) - f(g, u - e)) / (2 * e), rtol=1e-7, atol=1e-9)
    torch_act = torch.nn.functional.silu(g) if kind == "silu" else torch.nn.functional.gelu(g, approximate="tanh")
    assert torch.allclose(h, torch_act * u, rtol=1e-12, atol=1e-14)


def test_norm_gradients_against_differences():
    gen = torch.Generator().manual_seed(0)
    r = torch.randn(3, 37, generator=gen, dtype=torch.float64)
    w = 1 + 0.3 * torch.randn(37, generator=gen, dtype=torch.float64)
    dy = torch.randn(3, 37, generator=gen, dtype=torch.float64)
    dres = torch.randn(3, 37, generator=gen, dtype=torch.float64)
    _, rstd, _ = ref.norm(r, None, w, 1e-5)
    dx, dw = ref.norm_bwd(dy, r, w, rstd, dres)
    loss = lambda rr, ww: (dy * ref.norm(rr, None, ww, 1e-5)[2]).sum() + (dres * rr).sum()  # noqa: E731
    e = 1e-6
    for i, j in ((0, 0), (1, 17), (2, 36)):
        d = torch.zeros_like(r)
        d[i, j] = e
        assert abs((loss(r + d, w) - loss(r - d, w)) / (2 * e) - dx[i, j]) < 1e-7
        d = torch.zeros_like(w)
        d[j] = e
        assert abs((loss(r, w + d) - loss(r, w - d)) / (2 * e) - dw[j]) < 1e-7


# --------------------------------------------------------------------------------------------
# refusals: nothing below reaches the device
# --------------------------------------------------------------------------------------------
P = 1 << 20          # an "aligned pointer"; every call must fail before using it
INVALID, UNSUPPORTED, WORKSPACE, OK = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE, binding.OK


def blk(codes=P, ld=256, scale=P, ld_scale=2, tile=1):
    return ctypes.byref(binding._Blocks(codes, ld, scale, ld_scale, tile))


BAD_BLOCKS = [(dict(codes=None), INVALID), (dict(codes=P + 8), INVALID), (dict(ld=248), INVALID), (dict(ld=192), INVALID),
              (dict(scale=None), INVALID), (dict(scale=P + 2), INVALID), (dict(ld_scale=1), INVALID), (dict(tile=64), INVALID), (dict(tile=0), INVALID)]
RNE = ctypes.byref(binding.BLOCK_RNE.c())


def bad_rounding():
    base = dict(bits=8, scale=binding.PER_BLOCK, round=binding.RNE, format=binding.GRID_E4M3)
    for change, status in ((dict(bits=7), UNSUPPORTED), (dict(scale=binding.PER_ROW), UNSUPPORTED), (dict(scale=9), INVALID),
                           (dict(round=binding.RTN), UNSUPPORTED), (dict(round=7), INVALID), (dict(format=binding.GRID_INT), UNSUPPORTED),
                           (dict(format=5), INVALID)):
        yield ctypes.byref(binding.QSpec(**{**base, **change}).c()), status
    yield None, INVALID


def test_quantize_blocks_refusals(L):
    f = lambda x=P, dt=0, r=8, c=200, ld=200, q=RNE, rm=None, tr=None, s=None: int(L.srq_quantize_blocks(x, dt, r, c, ld, q, rm or blk(), tr, s, None))  # noqa: E731
    assert f(x=None) == f(x=P + 4) == f(dt=2) == f(r=-1) == f(c=-1) == f(ld=199) == f(s=P + 1) == INVALID
    assert int(L.srq_quantize_blocks(P, 0, 8, 200, 200, RNE, None, None, None, None)) == INVALID        # no layout
    for change, status in BAD_BLOCKS:
        assert f(rm=blk(**change)) == status, change
    for q, status in bad_rounding():
        assert f(q=q) == status
    assert f(tr=blk(ld=0)) == INVALID
    assert f(r=0) == OK and f(c=0, ld=0) == OK
    g = lambda x, rm: int(L.srq_requantize_blocks(x, 8, 200, RNE, rm, None, None, None))  # noqa: E731
    assert g(None, blk()) == INVALID and g(blk(), None) == INVALID
    for change, status in BAD_BLOCKS:
        assert g(blk(**change), blk()) == status, change


def test_gemm_blocks_refusals(L):
    def f(a=None, b=None, m=8, n=16, k=200, out=P, dt=0, ldo=16, acc=0, s=None):
        return int(L.srq_gemm_blocks(a or blk(), b or blk(), m, n, k, out, dt, ldo, acc, s, None))
    assert f(out=None) == f(m=-1) == f(n=-1) == f(k=-1) == f(ldo=15) == f(dt=2) == f(acc=2) == f(out=P + 2) == f(s=P + 2) == INVALID
    assert f(acc=1, dt=1) == UNSUPPORTED                       # running sums stay in binary32
    for change, status in BAD_BLOCKS:
        assert f(a=blk(**change)) == status and f(b=blk(**change)) == status, change
    assert f(m=0) == OK and f(n=0) == OK and f(k=0, acc=1) == OK


def test_norm_refusals(L):
    def f(x=P, ldx=200, res=P, ldr=200, dt=1, w=P, wdt=1, rows=8, cols=200, eps=1e-5, q=RNE, y=blk(), yo=None, ldy=200, ro=P, ld=200, rstd=P, s=None):
        return int(L.srq_rmsnorm_fwd(x, ldx, res, ldr, dt, w, wdt, rows, cols, eps, q, y, yo, ldy, ro, ld, rstd, s, None))
    for bad in (dict(x=None), dict(w=None), dict(rows=-1), dict(cols=-1), dict(dt=3), dict(wdt=3), dict(eps=-1.0), dict(eps=float("nan")),
                dict(ldx=199), dict(ldr=199), dict(ld=199), dict(yo=P, ldy=199), dict(x=P + 8), dict(res=P + 8), dict(w=P + 8), dict(ro=P + 8),
                dict(rstd=P + 2), dict(s=P + 2), dict(y=None)):
        assert f(**bad) == INVALID, bad
    assert f(y=blk(tile=128)) == UNSUPPORTED
    for q, status in bad_rounding():
        assert f(q=q) == status
    assert f(rows=0) == OK
    need = binding.srq_rmsnorm_workspace_bytes(600, 200)
    assert need == 512 * 256 * 4 and binding.srq_rmsnorm_workspace_bytes(3, 64) == 3 * 64 * 4 and binding.srq_rmsnorm_workspace_bytes(-1, 2) == 0

    def b(dy=P, ldy=200, r=P, ldr=200, d=None, ldd=200, dt=0, w=P, wdt=0, rstd=P, rows=600, cols=200, dx=P, ldx=200, dw=P, ws=P, nb=need):
        return int(L.srq_rmsnorm_bwd(dy, ldy, r, ldr, d, ldd, dt, w, wdt, rstd, rows, cols, dx, ldx, dw, ws, nb, None))
    for bad in (dict(dy=None), dict(r=None), dict(w=None), dict(rstd=None), dict(rows=-1), dict(cols=-1), dict(dt=2), dict(wdt=2), dict(dx=None, dw=None),
                dict(ldy=1), dict(ldr=1), dict(d=P, ldd=1), dict(ldx=1), dict(dy=P + 4), dict(d=P + 4), dict(dx=P + 4), dict(dw=P + 2), dict(ws=None), dict(ws=P + 64)):
        assert b(**bad) == INVALID, bad
    assert b(nb=need - 1) == WORKSPACE
    assert b(rows=0, dw=None, ws=None) == OK


def test_glu_refusals(L):
    def f(x=None, wg=None, wu=None, t=8, n=200, k=200, act=0, h=blk(), ho=None, hdt=0, ldh=200, gate=None, up=None, s=None):
        return int(L.srq_glu_fwd(x or blk(), wg or blk(), wu or blk(), t, n, k, act, h, ho, hdt, ldh, gate, up, s, None))
    for bad in (dict(t=-1), dict(n=-1), dict(k=0), dict(act=2), dict(h=None), dict(wg=blk(tile=128)), dict(ho=P, hdt=4), dict(ho=P, ldh=199), dict(ho=P + 4), dict(s=P + 1)):
        assert f(**bad) == INVALID, bad
    for change, status in BAD_BLOCKS:
        for name in ("x", "wg", "wu", "h", "gate", "up"):
            assert f(**{name: blk(**change)}) == status, (name, change)
    for name in ("h", "gate", "up"):
        assert f(**{name: blk(tile=128)}) == UNSUPPORTED
    assert f(t=0) == OK and f(n=0) == OK

    def b(dh=P, dt=0, ld=200, gate=None, up=None, t=200, n=200, act=1, q=RNE, dg=blk(), s=None, **more):
        return int(L.srq_glu_bwd(dh, dt, ld, gate or blk(), up or blk(), t, n, act, q, dg, *(more.get(k) for k in ("du", "dg_t", "du_t", "h_t")), s, None))
    for bad in (dict(dh=None), dict(dh=P + 4), dict(dt=2), dict(ld=199), dict(t=-1), dict(n=-1), dict(act=-1), dict(dg=None), dict(s=P + 2)):
        assert b(**bad) == INVALID, bad
    for change, status in BAD_BLOCKS:
        for name in ("gate", "up", "dg", "du", "dg_t", "du_t", "h_t"):
            assert b(**{name: blk(**change)}) == status, (name, change)
    for name in ("gate", "up", "dg", "h_t"):
        assert b(**{name: blk(tile=128)}) == UNSUPPORTED
    for q, status in bad_rounding():
        assert b(q=q) == status
    assert b(t=0) == OK and b(n=0) == OK


def test_null_pointers_are_for_operands_without_elements(L):
    none = lambda tile=1: ctypes.byref(binding._Blocks(None, 208, None, 2, tile))  # noqa: E731
    for r, c in ((0, 200), (8, 0), (0, 0)):
        assert int(L.srq_quantize_blocks(None, 0, r, c, 200, RNE, none(), none(128), None, None)) == OK
        assert int(L.srq_requantize_blocks(none(), r, c, RNE, none(), none(), None, None)) == OK
        assert int(L.srq_gemm_blocks(none(), none(), r, c, 0, None, 0, 200, 0, None, None)) == OK
        assert int(L.srq_rmsnorm_fwd(None, 200, None, 200, 1, None, 1, r, c, 1e-5, RNE, none(), None, 200, None, 200, None, None, None)) == OK
        assert int(L.srq_rmsnorm_bwd(None, 200, None, 200, None, 200, 0, None, 0, None, r, c, None, 200, None, None, 0, None)) == OK
        assert int(L.srq_glu_fwd(none() if r == 0 else blk(), none() if c == 0 else blk(), none() if c == 0 else blk(), r, c, 200, 0, none(), None, 0, 200, none(), none(), None, None)) == OK
        assert int(L.srq_glu_bwd(None, 0, 200, none(), none(), r, c, 0, RNE, none(), none(), none(), none(), none(), None, None)) == OK
        # the rest of the arguments is checked as ever
        assert int(L.srq_quantize_blocks(None, 7, r, c, 200, RNE, none(), None, None, None)) == INVALID
        assert int(L.srq_quantize_blocks(None, 0, r, c, 200, RNE, None, None, None, None)) == INVALID
        assert int(L.srq_gemm_blocks(none(), none(64), r, c, 0, None, 0, 200, 0, None, None)) == INVALID
        assert int(L.srq_glu_bwd(None, 0, 200, none(), none(128), r, c, 0, RNE, none(), None, None, None, None, None, None)) == UNSUPPORTED
    # an operand that has elements needs its pointers even where the result has none, or where the contraction is empty
    assert int(L.srq_gemm_blocks(none(), none(), 0, 8, 200, None, 0, 200, 0, None, None)) == INVALID
    assert int(L.srq_gemm_blocks(none(), none(), 8, 8, 0, None, 0, 200, 0, None, None)) == INVALID


def test_block_modes_stay_out_of_the_other_entry_points(L):
    for q in (binding.QSpec(scale=binding.PER_BLOCK), binding.QSpec(round=binding.RNE)):
        assert int(L.sr_quantize(P, 0, 8, 8, 8, ctypes.byref(q.c()), P, 8, P, None, 0, None, P, 1 << 20, None)) == INVALID


def test_binding_checks_shapes_before_the_call():
    cpu = torch.zeros((4, 16), dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        binding.Blocks(cpu, torch.zeros((4, 1))).c()
    with pytest.raises(ValueError):
        binding.srq_gemm_blocks(binding.Blocks(cpu, torch.zeros((4, 1))), binding.Blocks(cpu, torch.zeros((4, 1))), torch.zeros((4, 5)))


def test_the_adding_warps_meet_after_a_wait():
    """Their waits are loops that a lane leaves by itself, and what follows is tcgen05.ld.sync.aligned, which takes a
    converged warp.  The wait must therefore end by bringing the lanes together, on every path through it."""
    text = open(os.path.join(os.path.dirname(binding.__file__), "csrc", "gemm_blocks.cu")).read()
    start = text.index("void wait_or_abort(")
    body = text[text.index("{", start) + 1:text.index("\n}\n", start)]
    assert "return" not in body and body.rstrip().endswith("__syncwarp();")
    # and they have no other way to wait: what lies between a wait and the loads after it
    calls = [m.start() for m in re.finditer(r"wait_or_abort\((?!uint32_t)", text)]
    assert len(calls) == 3                       # step sizes and sums (CTA pairs), sums (few tokens)
    for load in re.finditer(r"tmem_ld(?:16|32)\((?:tb|taddr)", text):
        before = text[max(c for c in calls if c < load.start()):load.start()]
        assert "mbar_wait(" not in before and "try_wait" not in before


def test_kernels_launched_early_do_not_read_through_the_read_only_path():
    """A programmatic dependent is running while its predecessor writes what it will read after its wait, so those reads
    must be ordinary ones: ld.global.nc (__ldg) takes data that nobody writes for as long as the kernel runs."""
    src = os.path.join(os.path.dirname(binding.__file__), "csrc")
    for name in ("blocks.cuh", "gemm_blocks.cu", "quantize_blocks.cu", "rmsnorm.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(src, name)).read())
        assert not re.search(r"__ldg\s*\(|ld\.global\.nc", text), name
