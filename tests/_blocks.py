"""Plain 64-bit implementations of the block-scaled operators, written from their definitions, and the
bounds the tests hold the kernels to.  Used by the tests only."""
import math

import numpy as np
import torch

import _independent as ind

BLK = 128
ULP = 2.0 ** -24           # unit roundoff of binary32


# --------------------------------------------------------------------------------------------
# the quantizer, exactly
# --------------------------------------------------------------------------------------------
def steps(m):
    """Step size and reciprocal (binary32, the reciprocal rounded toward zero) of blocks with absmax m (float32)."""
    m = np.asarray(m, dtype=np.float32)
    with np.errstate(divide="ignore", over="ignore"):
        q = 448.0 / m.astype(np.float64)
        inv = q.astype(np.float32)
    inv = np.where(inv.astype(np.float64) > q, np.nextafter(inv, np.float32(0)), inv).astype(np.float32)
    dead = m <= np.float32(7.0 * 2.0 ** -122)
    return np.where(dead, np.float32(0), m / np.float32(448)).astype(np.float32), np.where(dead, np.float32(0), inv).astype(np.float32)


def quantize(x, tile_rows=1, thresholds=None):
    """(codes uint8, step sizes float32) of a float32 matrix; thresholds: u24 of every element for SR."""
    x = np.asarray(x, dtype=np.float32)
    r, c = x.shape
    nr, nc = -(-r // tile_rows), -(-c // BLK)
    full = np.zeros((nr * tile_rows, nc * BLK), dtype=np.float32)
    full[:r, :c] = np.abs(x)
    m = full.reshape(nr, tile_rows, nc, BLK).max(axis=(1, 3))
    step, inv = steps(m)
    spread = np.repeat(np.repeat(inv, tile_rows, 0)[:r], BLK, 1)[:, :c]
    t = (x * spread).astype(np.float32)
    if thresholds is None:
        codes = torch.from_numpy(t).to(torch.float8_e4m3fn)
    else:
        t64 = t.astype(np.float64)
        e = np.maximum(np.frexp(np.abs(t64))[1] - 1, -6)
        e = np.where(t64 == 0, -6, e)
        u = t64 * 2.0 ** (3 - e)
        f = np.floor(u)
        q = f + (np.asarray(thresholds, dtype=np.float64) * 2.0 ** -24 < u - f)
        codes = torch.from_numpy((q * 2.0 ** (e - 3) + 0.0).astype(np.float32)).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).numpy(), step


def thresholds(q, rows, cols):
    return ind.thresholds_u24(q.seed, q.tensor_id, q.index_offset, rows, cols)


def values(codes, step, tile_rows=1):
    """The numbers block codes stand for (float64); torch tensors on any device."""
    r, c = codes.shape
    s = step.double().repeat_interleave(tile_rows, 0)[:r].repeat_interleave(BLK, 1)[:, :c]
    return codes.contiguous().view(torch.float8_e4m3fn).double() * s


def _spacing(t):
    """Distance of neighbouring E4M3 numbers at |t|."""
    return torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))).clamp(min=-6) - 3)


def check_coded(codes, step, ref, err, what):
    """Codes against the real numbers ref, of which the kernel knew each to within err (both float64,
    [rows, cols], blocks along the columns): step sizes are the block's maximum over 448, every number is
    within half a step of the grid."""
    r, c = ref.shape
    nb = -(-c // BLK)
    pad = lambda v: torch.nn.functional.pad(v, (0, nb * BLK - c)).view(r, nb, BLK)  # noqa: E731
    top, slack = pad(ref.abs()).amax(2), pad(err).amax(2)
    d = step.double()[:, :nb]
    bad = (d * 448 - top).abs() > slack + 4 * ULP * top + 1e-38
    assert not bad.any(), f"{what}: step sizes off at {bad.nonzero()[0].tolist()}"
    dd = d.repeat_interleave(BLK, 1)[:, :c]
    got = codes.contiguous().view(torch.float8_e4m3fn).double() * dd
    safe = dd.clamp(min=1e-300)
    half = 0.5 * _spacing((ref.abs() + err) / safe) * dd
    bad = (got - ref).abs() > half * (1 + 2.0 ** -20) + err + 8 * ULP * ref.abs()
    assert not bad.any(), f"{what}: {int(bad.sum())} codes off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {ref[bad][0]}"


# --------------------------------------------------------------------------------------------
# the product
# --------------------------------------------------------------------------------------------
def product(a, b):
    """(A B^T, bound of the kernel's binary32 error): 128 products added on the tensor core (each addition may
    truncate: 2 units), one scaling and one addition per block, all relative to the sum of magnitudes."""
    ref = a @ b.t()
    kb = -(-a.shape[1] // BLK)
    return ref, (2 * BLK + 2 * kb + 16) * ULP * (a.abs() @ b.abs().t())


# --------------------------------------------------------------------------------------------
# the gated activations
# --------------------------------------------------------------------------------------------
def act(g, kind):
    """act(g), act'(g) and the sum of the magnitudes of act's two terms (what rounding acts on)."""
    if kind == "silu":
        p, dz = torch.sigmoid(g), torch.ones_like(g)
    else:
        k = math.sqrt(2.0 / math.pi)
        p = torch.sigmoid(2.0 * k * (g + 0.044715 * g ** 3))
        dz = 2.0 * k * (1.0 + 3.0 * 0.044715 * g ** 2)
    a = g * p
    tail = a * (1.0 - p) * dz
    return a, p + tail, p + tail.abs()


# e^-z by the fast exponential carries a relative error of about |z| + 2 units, which the logistic function passes on
# times 1 - p <= 1 while it matters (|z| < 90); two roundings each for the rest
ACT_ERR = 128 * ULP


def glu(x, wg, wu, kind):
    """(g, u, h) with error bounds."""
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    a, _, _ = act(g, kind)
    h = a * u
    eh = 1.2 * (eg * u.abs() + a.abs() * eu + eg * eu) + ACT_ERR * h.abs()
    return (g, eg), (u, eu), (h, eh)


def glu_bwd(dh, g, u, kind):
    a, da, mag = act(g, kind)
    dg, du, h = dh * u * da, dh * a, a * u
    return (dg, ACT_ERR * (dh * u).abs() * mag), (du, ACT_ERR * du.abs()), (h, ACT_ERR * h.abs())


# --------------------------------------------------------------------------------------------
# the norm
# --------------------------------------------------------------------------------------------
def norm(x, residual, w, eps):
    r = x if residual is None else x + residual
    rstd = 1.0 / torch.sqrt(r.square().mean(1) + eps)
    return r, rstd, r * rstd[:, None] * w


def norm_bwd(dy, r, w, rstd, d_residual):
    n = r * rstd[:, None]
    wdy = dy * w
    dx = rstd[:, None] * (wdy - n * (wdy * n).mean(1, keepdim=True))
    if d_residual is not None:
        dx = dx + d_residual
    return dx, (dy * n).sum(0)


def depth(cols):
    """Additions one value can pass through in a row's sum: at most 1024 threads, eight values a time, then a tree."""
    return 8 * -(-cols // 256) + 40 if cols <= 8192 else 8 * -(-cols // 8192) + 8 * 4 + 40
