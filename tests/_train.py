"""Plain implementations, in 64 bits unless they are exact in 32, of the operators at the ends of a training step, and the bounds
the tests hold the kernels to.  Used by the tests only."""
import math

import numpy as np
import torch

import _independent as ind

BLK = 128
ULP = 2.0 ** -24                 # unit roundoff of binary32
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


# --------------------------------------------------------------------------------------------
# embedding
# --------------------------------------------------------------------------------------------
def embed(table, ids, scale, out_dtype):
    """Exact: one product in binary32, rounded once more where the output is narrower."""
    ok = (ids >= 0) & (ids < table.shape[0])
    rows = table.float()[ids.clamp(0, max(0, table.shape[0] - 1)).long()] if table.shape[0] else torch.zeros((len(ids), table.shape[1]), device=table.device)
    return torch.where(ok[:, None], rows * torch.tensor(scale, dtype=torch.float32, device=table.device), 0.0).to(out_dtype)


def embed_bwd(dout, ids, rows, scale):
    """(gradient in 64 bits, bound): n terms are added in binary32 (n - 1 roundings and one for each of at most 1184 parts), the
    scale rounds twice (itself and the product)."""
    ok = (ids >= 0) & (ids < rows)
    i, x = ids[ok].long(), dout[ok].double()
    zero = lambda: torch.zeros((rows, dout.shape[1]), dtype=torch.float64, device=dout.device)  # noqa: E731
    total, size = zero().index_add_(0, i, x), zero().index_add_(0, i, x.abs())
    n = torch.zeros(rows, dtype=torch.float64, device=dout.device).index_add_(0, i, torch.ones(len(i), dtype=torch.float64, device=dout.device))
    return total * scale, (n + 1184 * (n > 8) + 3)[:, None] * ULP * size * abs(scale)


# --------------------------------------------------------------------------------------------
# losses on the logits
# --------------------------------------------------------------------------------------------
def logprob(x, targets, temperature=1.0):
    """(logp, lse, p, bound of logp and lse, relative bound of p) in 64 bits; rows that do not count are 0.

    Bounds: an exponential carries 2 units of its own and those of its argument (difference, factor, product), 3 units of |z - max|,
    which e^-|z - max| brings below 2 on the sum; a thread adds at most classes / 128 / 2 terms in a row and 16 more in the
    joins, each of which rounds three times; log and the last differences a few units of their results."""
    z = x.double() / temperature
    counts = (targets >= 0) & (targets < x.shape[1])
    t = targets.clamp(0, x.shape[1] - 1).long()[:, None]
    m = z.max(1, keepdim=True).values
    lse = torch.logsumexp(z, 1)
    zt = z.gather(1, t)[:, 0]
    zero = torch.zeros_like(lse)
    sum_err = (x.shape[1] / 256 + 64) * ULP
    err = sum_err + 4 * ULP * ((zt - m[:, 0]).abs() + lse.abs() + m[:, 0].abs() + 1)
    rel = sum_err + ULP * (8 + 4 * (z - m).abs().nan_to_num(posinf=0.0))
    return torch.where(counts, zt - lse, zero), torch.where(counts, lse, zero), torch.exp(z - lse[:, None]), err, rel, counts


def dlogits(p, rel, targets, counts, c, c_err, temperature=1.0):
    """(gradient at the logits, bound before its rounding to the output's type)."""
    c, c_err = torch.where(counts, c, 0.0) / temperature, torch.where(counts, c_err, 0.0) / temperature
    d = -c[:, None] * p
    err = (c.abs()[:, None] * (rel + 6 * ULP) + c_err[:, None]) * p
    t = targets.clamp(0, p.shape[1] - 1).long()[:, None]
    d.scatter_add_(1, t, c[:, None])
    err.scatter_add_(1, t, (c_err + 4 * ULP * c.abs())[:, None])
    return d, err


def policy(logp, old, adv, weight, ref, lo, hi, kl):
    """(row_loss, dlogp) in 64 bits."""
    rho = torch.exp(logp - old)
    a, b = rho * adv, rho.clamp(1 - lo, 1 + hi) * adv
    loss, c = -torch.minimum(a, b), torch.where(a <= b, -a, 0.0)
    if ref is not None:
        d = ref - logp
        loss, c = loss + kl * (torch.expm1(d) - d), c - kl * torch.expm1(d)
    return weight * loss, weight * c


def policy_bounds(logp, err, old, adv, weight, ref, kl):
    """Bounds of row_loss and dlogp for a logp that is off by err: the exponentials pass it on as a relative error, with 4 units of
    their own (the argument's rounding included, per unit of the argument), and a few roundings follow."""
    rho = torch.exp(logp - old)
    e = err + ULP * (8 + (logp - old).abs() + logp.abs())
    loss = rho * adv.abs() * e
    c = loss.clone()
    if ref is not None:
        d = ref - logp
        f = err + ULP * (8 + d.abs() + logp.abs())
        loss = loss + kl * (torch.exp(d) * f + f + 4 * ULP * (torch.expm1(d).abs() + d.abs()))
        c = c + kl * (torch.exp(d) * f + 4 * ULP * torch.expm1(d).abs())
    return weight.abs() * (loss * 1.01 + 1e-30), weight.abs() * (c * 1.01 + 1e-30)


def preference(diff, offsets, beta, smoothing):
    """(pair_loss, h, gradient of their mean at every row's logp) from logp - ref (0 where a row does not count)."""
    o = offsets.tolist()
    s = torch.stack([diff[a:b].sum() for a, b in zip(o, o[1:])]) if len(o) > 1 else diff.new_zeros(0)
    h = beta * (s[0::2] - s[1::2])
    pair = -(1 - smoothing) * torch.nn.functional.logsigmoid(h) - smoothing * torch.nn.functional.logsigmoid(-h)
    dh = (smoothing - torch.sigmoid(-h)) * beta / max(1, len(h))
    c = torch.zeros_like(diff)
    for k, (a, b) in enumerate(zip(o, o[1:])):
        c[a:b] = dh[k // 2] * (1 if k % 2 == 0 else -1)
    return pair, h, c


# --------------------------------------------------------------------------------------------
# AdamW
# --------------------------------------------------------------------------------------------
def words(n, seed, tensor_id):
    """Philox words of elements 0 .. n - 1 (uint64 holding 32 bits)."""
    i = np.arange(n, dtype=np.uint64)
    j = i >> np.uint64(2)
    w = ind.philox_np(j & ind.MASK, j >> ind.S32, np.full_like(j, tensor_id & 0xFFFFFFFF), np.full_like(j, (tensor_id >> 32) & 0xFFFFFFFF),
                      seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    return np.take_along_axis(np.stack(w), (i & np.uint64(3)).astype(np.int64)[None], 0)[0]


def grid_value(code, mantissa):
    """The number a code without its sign stands for: exponent bias 7, `mantissa` bits."""
    code = np.asarray(code, dtype=np.int64)
    e, m = code >> mantissa, (code & ((1 << mantissa) - 1)).astype(np.float64)
    return np.where(e == 0, m * 2.0 ** (-6 - mantissa), (2.0 ** mantissa + m) * 2.0 ** (e - 7.0 - mantissa))


def block_steps(amax, top):
    """Step size (a product with 1 / top) and reciprocal, the latter rounded toward zero, of blocks with the absmax `amax` (float32)."""
    amax = np.asarray(amax, dtype=np.float32)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        q = top / amax.astype(np.float64)
        inv = q.astype(np.float32)
        dead = (amax == 0) | np.isinf(np.float32(top) / amax)
        inv = np.where(inv.astype(np.float64) > q, np.nextafter(inv, np.float32(0)), inv).astype(np.float32)
        step = (amax * np.float32(1.0 / top)).astype(np.float32)
    return np.where(dead, np.float32(0), step), np.where(dead, np.float32(0), inv)


def encode(x, u, top, mantissa):
    """(codes, steps) of x (float32, any length, blocks of 128) with thresholds u in [0, 2^16): the magnitude of x / step goes to the
    grid's next number above it if the part cut off, in units of the grid's spacing, and (u + 1/2) / 2^16 add up to 1."""
    n = len(x)
    pad = np.zeros(-(-n // BLK) * BLK, dtype=np.float32)
    pad[:n] = x
    amax = np.abs(pad).reshape(-1, BLK).max(1)
    step, inv = block_steps(amax, top)
    t = np.abs(x * np.repeat(inv, BLK)[:n]).astype(np.float64)
    # subnormal numbers of the grid: the quotient is held to 2^-29 (rounded to nearest even), 20 bits below the spacing 2^-9
    t = np.where(t < 2.0 ** -6, np.rint(t * 2.0 ** 29) * 2.0 ** -29, t)
    e = np.where(t > 0, np.maximum(np.frexp(t)[1] - 1, -6), -6)
    spacing = 2.0 ** (e - mantissa)
    # exact: the quotient has at most 20 bits below the spacing
    q = np.floor(t / spacing + (np.asarray(u, dtype=np.float64) + 0.5) * 2.0 ** -16)
    code = np.rint(q + np.maximum(e + 6, 0) * 2.0 ** mantissa).astype(np.int64)       # q in [2^mantissa, 2^(mantissa+1)] from e = -6 on
    return code, step


def moments(m, v, g, beta1, beta2):
    """New moments in binary32, every product and sum rounded once."""
    f = np.float32
    m = (m * f(beta1)).astype(f) + (g * f(1 - beta1)).astype(f)
    v = (v * f(beta2)).astype(f) + ((g * g).astype(f) * f(1 - beta2)).astype(f)
    return m.astype(f), v.astype(f)


def weight(p, m, v, h, t):
    """(new weight in 64 bits, bound).  Root and reciprocal are approximations (2 units each), the root's argument is the rounded v,
    eps, the bias corrections and the rates are rounded once each, and so are the products."""
    p, m, v = (a.astype(np.float64) for a in (p, m, v))
    b1, b2 = -math.expm1(t * math.log(h["beta1"])) if h["beta1"] else 1.0, -math.expm1(t * math.log(h["beta2"])) if h["beta2"] else 1.0
    u = h["lr"] / b1 * m / (np.sqrt(v / b2) + h["eps"])
    return p * (1 - h["lr"] * h["weight_decay"]) - u, ULP * (5 * np.abs(p) + 24 * np.abs(u)) + 1e-45


def cut_bf16(x, u):
    """bfloat16 of float32 x, cut after the threshold u in [0, 2^16) was added to the bits below it (as float32)."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64) + np.asarray(u, dtype=np.uint64)
    return ((b >> np.uint64(16)) << np.uint64(16)).astype(np.uint32).view(np.float32)
