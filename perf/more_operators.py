"""The two ends of a language model's training step and its update, as they are measured.

Operators around the layers that this repository trains with few bits:

  embed       out[t] = scale * table[id_t]; an id below zero is padding and gives zeros
  embed_bwd   dtable[v] = scale * sum of dout[t] over the tokens t with id_t = v
  policy      clipped policy loss with a KL term on the logits, and the gradient at the logits
  preference  paired log ratios of chosen and rejected answers on the logits, and the gradient at the logits
  adamw       one step over many tensors: moments in 32 bits, or in 8 bits with a step size per 128 values, weights in
              binary32 or in bfloat16 with stochastic rounding

`run` computes a case in plain torch operations where `own` is false, and through the library where it is true.  `exact`
computes it from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

BLK = 128                        # values per step size of an 8-bit moment
M_MAX, V_MAX = 448.0, 496.0      # largest numbers of the two 8-bit grids
CLIP, KL_COEF = 0.2, 0.05
BETA, SMOOTHING = 0.1, 0.05
ADAMW = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "weight_decay": 0.1, "step": 1000}
SEED, TENSOR_ID = 11, 500


def listed():
    return [
        # the next token of four generated answers on its way into the first layer
        {"name": "embed 4 tokens", "op": "embed", "t": 4, "v": 32000, "d": 2048, "dtype": "bf16", "scale": 1.0},
        # a training batch of 16 sequences
        {"name": "embed batch", "op": "embed", "t": 16384, "v": 32000, "d": 4096, "dtype": "bf16", "scale": 64.0},
        # its gradient at a 2048-wide model, kept in 32 bits for the optimizer
        {"name": "embed gradient", "op": "embed_bwd", "t": 16384, "v": 32000, "d": 2048, "dtype": "bf16", "scale": 1.0},
        # a ragged batch on a vocabulary of odd size, 768 wide, everything in 32 bits
        {"name": "embed gradient odd", "op": "embed_bwd", "t": 5003, "v": 50257, "d": 768, "dtype": "f32", "scale": 27.712812921102035},
        # the last tokens of a few short answers
        {"name": "policy few tokens", "op": "policy", "t": 64, "v": 32000, "dtype": "bf16", "masked": 0.0, "ref": True},
        # 32-bit logits of a vocabulary whose rows start anywhere, no reference model
        {"name": "policy odd", "op": "policy", "t": 1021, "v": 50257, "dtype": "f32", "masked": 0.1, "ref": False},
        # a micro-batch of answers on a large vocabulary, an eighth of the rows being prompts
        {"name": "policy batch", "op": "policy", "t": 4096, "v": 131072, "dtype": "bf16", "masked": 0.125, "ref": True},
        # two short pairs on 32-bit logits
        {"name": "preference two pairs", "op": "preference", "pairs": 2, "length": 40, "v": 32000, "dtype": "f32"},
        # sixteen pairs of answers of different length on a vocabulary of odd size
        {"name": "preference batch", "op": "preference", "pairs": 16, "length": 256, "v": 50257, "dtype": "bf16"},
        # the norms' weights of a small model, in a group of their own without weight decay
        {"name": "adamw norms", "op": "adamw", "layers": 18, "features": 2048, "hidden": 0, "dtype": "f32", "grad": "f32", "bits": 32},
        # one layer, everything in 32 bits
        {"name": "adamw layer", "op": "adamw", "layers": 1, "features": 2048, "hidden": 5632, "dtype": "f32", "grad": "f32", "bits": 32},
        # eight layers with weights and gradients in bfloat16 and moments in 8 bits
        {"name": "adamw 8 bits", "op": "adamw", "layers": 8, "features": 2048, "hidden": 5632, "dtype": "bf16", "grad": "bf16", "bits": 8},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, uniform over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_bwd", "policy", "preference", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    even = rng.random() < 0.5                  # half of the cases have the usual sizes, half of them odd ones
    size = lambda lo, hi, m: -(-_spread(rng, lo, hi) // m) * m if even else _spread(rng, lo, hi)  # noqa: E731
    if op in ("embed", "embed_bwd"):
        return {"op": op, "t": _spread(rng, 1, 16384), "v": _spread(rng, 200, 50000), "d": min(4096 if op == "embed" else 2048, size(64, 4096, 128)),
                "dtype": dtype, "scale": rng.choice([1.0, 45.254833995939045])}
    if op == "policy":
        v = min(131072, size(1000, 131072, 64))
        return {"op": op, "t": _spread(rng, 1, max(2, min(8192, 2 ** 29 // (v * _bytes(dtype))))), "v": v, "dtype": dtype,
                "masked": rng.choice([0.0, 0.2, 0.6]), "ref": rng.random() < 0.5}
    if op == "preference":
        v = min(65536, size(1000, 65536, 64))
        length = _spread(rng, 1, 500)
        return {"op": op, "pairs": _spread(rng, 1, max(1, min(64, 2 ** 26 // (v * length)))), "length": length, "v": v, "dtype": dtype}
    features, hidden = size(64, 2048, 64), rng.choice([0, 1, 1])
    hidden *= _spread(rng, features, int(2.75 * features))
    layers = _spread(rng, 1, 40) if not hidden else _spread(rng, 1, max(1, min(8, 50_000_000 // (features * (features + hidden)))))
    return {"op": op, "layers": layers, "features": features, "hidden": hidden, "dtype": dtype, "grad": rng.choice([dtype, "f32"]),
            "bits": rng.choice([8, 32])}


def _blocks(n):
    return (n + BLK - 1) // BLK


def _bytes(name):
    return {"f32": 4, "bf16": 2}[name]


def _distinct(case):
    """Expected number of different ids among the tokens (_ids below draws them log-uniformly)."""
    k = np.arange(1, case["v"] + 1, dtype=np.float64)
    p = np.log1p(1.0 / k) / math.log(case["v"] + 1)
    return float(-np.expm1(_tokens(case) * np.log1p(-p)).sum()) if case["v"] > 1 else 1.0


def _tokens(case):
    """Tokens that are not padding."""
    return case["t"] - case["t"] // 20


def _rows(case):
    """Rows of a policy case that count."""
    return case["t"] - int(case["t"] * case["masked"])


def _lengths(case):
    """Lengths of the answers, chosen and rejected in turn: from half of case["length"] to one and a half times it."""
    n = case["length"]
    return [max(1, n // 2 + (i * 7919) % (n + 1)) for i in range(2 * case["pairs"])]


def _shapes(case):
    """Weights of a model's layers: fused query/key/value, output, gate, up and down projections and two norms; hidden = 0: the norms alone."""
    k, f = case["features"], case["hidden"]
    layer = [(k,), (k,)] + ([(k + k // 4, k), (k, k), (f, k), (f, k), (k, f)] if f else [])
    return layer * case["layers"]


def work(case):
    op, e = case["op"], _bytes(case["dtype"])
    if op == "embed":
        return {"bytes": case["t"] * (case["d"] * e + 8) + _distinct(case) * case["d"] * e, "flops": case["t"] * case["d"]}
    if op == "embed_bwd":
        return {"bytes": _tokens(case) * case["d"] * e + case["t"] * 8 + case["v"] * case["d"] * 4, "flops": _tokens(case) * case["d"]}
    if op == "policy":
        return {"bytes": (_rows(case) + case["t"]) * case["v"] * e + case["t"] * 4 * (7 if case["ref"] else 6), "flops": 8 * _rows(case) * case["v"]}
    if op == "preference":
        t = sum(_lengths(case))
        return {"bytes": 2 * t * case["v"] * e + t * 16, "flops": 8 * t * case["v"]}
    n = sum(math.prod(s) for s in _shapes(case))
    state = 4 if case["bits"] == 8 else 16
    return {"bytes": n * (2 * e + _bytes(case["grad"]) + state) + (16 * _blocks(n) if case["bits"] == 8 else 0), "flops": 15 * n}


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _ids(g, t, v, padding):
    """Tokens as text has them: the k-th most frequent about 1 / k as often as the first (log-uniform), numbered in no order; the
    last `padding` are padding."""
    rank = torch.exp(_rand(g, t).double() * math.log(v + 1)).long().sub_(1).clamp_(0, v - 1)
    ids = torch.randperm(v, generator=g, device="cuda")[rank]
    ids[t - padding:] = -1
    return ids


def _logits(g, t, v, dtype):
    """Logits of a trained model: a common part, a row's own, and one answer in each row that stands out."""
    x = _randn(g, t, v, std=2.0)
    x += _randn(g, 1, v, std=1.5)
    top = torch.randint(0, v, (t, 1), generator=g, device="cuda")
    x.scatter_add_(1, top, 8.0 + 3.0 * _randn(g, t, 1))
    other = torch.randint(0, v, (t, 1), generator=g, device="cuda")
    targets = torch.where(_rand(g, t, 1) < 0.7, top, other).view(-1)
    return x.to(_dtype(dtype)), targets


def _flat(case):
    """Sizes of the tensors and where each begins in one buffer (multiples of 128 values)."""
    sizes = [math.prod(s) for s in _shapes(case)]
    starts = np.concatenate([[0], np.cumsum([_blocks(n) * BLK for n in sizes])]).tolist()
    return sizes, starts


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], {"case": case}
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if op in ("embed", "embed_bwd"):
        t, v, d, dt = case["t"], case["v"], case["d"], _dtype(case["dtype"])
        s["ids"] = _ids(g, t, v, t // 20)
        if op == "embed":
            s["table"] = _randn(g, v, d, std=0.02).to(dt)
            s["out"] = torch.empty((t, d), dtype=dt, device="cuda")
        else:
            s["dout"] = _randn(g, t, d, std=1e-3).to(dt)
            s["dtable"] = torch.empty((v, d), device="cuda")
    elif op == "policy":
        t, v = case["t"], case["v"]
        s["logits"], s["targets"] = _logits(g, t, v, case["dtype"])
        s["dlogits"] = torch.empty_like(s["logits"])
        logp = _token_logp(s["logits"], s["targets"])
        s["old"] = logp + _randn(g, t, std=0.15)              # the policy that sampled the answers
        s["ref"] = logp + _randn(g, t, std=0.4) if case["ref"] else None
        s["advantage"] = _randn(g, t)
        w = torch.full((t,), 1.0 / max(1, _rows(case)), device="cuda")
        w[torch.randperm(t, generator=g, device="cuda")[_rows(case):]] = 0.0
        s["weight"] = w
        s["logp"], s["row_loss"] = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        s["loss"] = torch.empty(1, device="cuda")
    elif op == "preference":
        n = _lengths(case)
        t, v = sum(n), case["v"]
        s["logits"], s["targets"] = _logits(g, t, v, case["dtype"])
        s["dlogits"] = torch.empty_like(s["logits"])
        s["ref"] = _token_logp(s["logits"], s["targets"]) + _randn(g, t, std=0.3)
        s["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int64, device="cuda")
        s["logp"], s["pair_loss"] = torch.empty(t, device="cuda"), torch.empty(case["pairs"], device="cuda")
        s["loss"] = torch.empty(1, device="cuda")
    else:
        sizes, starts = _flat(case)
        total = starts[-1]
        real = torch.zeros(total, dtype=torch.bool, device="cuda")
        for n, i in zip(sizes, starts):
            real[i:i + n] = True
        # gradients differ in size from one row of 128 to the next and from step to step
        size = 1e-3 * torch.exp(_randn(g, total // BLK, 1)).expand(-1, BLK).reshape(-1)
        s["p"] = (_randn(g, total, std=0.02) * real).to(_dtype(case["dtype"]))
        s["g"] = (_randn(g, total) * size * real).to(_dtype(case["grad"]))
        m = _randn(g, total, std=0.25) * size * real
        v = (_randn(g, total).square() * 0.2 + 0.8) * size.square() * real
        if case["bits"] == 8:
            half = torch.full((total,), 32767, dtype=torch.int64, device="cuda")
            s["m"], s["m_scale"] = _code(m, half, M_MAX, 20)
            s["v"], s["v_scale"] = _code(v, half, V_MAX, 19)
        else:
            s["m"], s["v"] = m, v
    return s


def _token_logp(logits, targets):
    """log-probability of the targets, row by row in 32 bits (making inputs only)."""
    top = logits.max(1).values.float()
    total = torch.stack([torch.exp(x.float() - m).sum() for x, m in zip(logits, top)]) if logits.shape[0] <= 64 else \
        torch.cat([torch.exp(x.float() - m[:, None]).sum(1) for x, m in zip(logits.split(512), top.split(512))])
    return logits.gather(1, targets[:, None])[:, 0].float() - top - torch.log(total)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------- in the framework
def _run_own(s):
    import paper_2511_00874_b200 as srq
    case = s["case"]
    op = case["op"]
    if op == "embed":
        srq.srq_embedding_fwd(s["table"], s["ids"], s["out"], case["scale"], device_status=s["status"])
        return {"out": s["out"]}
    if op == "embed_bwd":
        if "ws" not in s:                      # a program allocates its workspace once
            s["ws"] = srq.new_workspace(srq.srq_embedding_workspace_bytes(case["t"], case["v"], case["d"]))
        srq.srq_embedding_bwd(s["dout"], s["ids"], s["dtable"], case["scale"], ws=s["ws"], device_status=s["status"])
        return {"dtable": s["dtable"]}
    if op == "policy":
        srq.srq_policy_loss(s["logits"], s["targets"], s["old"], s["advantage"], s["weight"], s["ref"], s["row_loss"], s["loss"], s["logp"],
                            s["dlogits"], clip_low=CLIP, clip_high=CLIP, kl_coef=KL_COEF, device_status=s["status"])
        return {n: s[n] for n in ("loss", "row_loss", "logp", "dlogits")}
    if op == "preference":
        if "ws" not in s:
            s["ws"] = srq.new_workspace(srq.srq_preference_workspace_bytes(s["logits"].shape[0]))
        srq.srq_preference_loss(s["logits"], s["targets"], s["ref"], s["offsets"], s["pair_loss"], s["loss"], s["logp"], s["dlogits"],
                                beta=BETA, label_smoothing=SMOOTHING, ws=s["ws"], device_status=s["status"])
        return {n: s[n] for n in ("loss", "pair_loss", "logp", "dlogits")}
    if "tensors" not in s:                     # a program lists its weights, gradients and moments once
        sizes, starts = _flat(case)
        part = lambda name, n, i: s[name][i:i + n]  # noqa: E731
        steps = lambda name, n, i: s[name][i // BLK:i // BLK + _blocks(n)] if case["bits"] == 8 else None  # noqa: E731
        s["tensors"] = srq.AdamTensors([srq.AdamTensor(part("p", n, i), part("g", n, i), part("m", n, i), part("v", n, i),
                                                       steps("m_scale", n, i), steps("v_scale", n, i)) for n, i in zip(sizes, starts)])
    srq.srq_adamw_step(s["tensors"], **ADAMW, round=srq.SR, seed=SEED, tensor_id=TENSOR_ID, device_status=s["status"])
    return _moments(s)


def _moments(s):
    """Weights and moments; of 8-bit moments the E4M3 numbers of the first, the codes of the second, and the step sizes."""
    if s["case"]["bits"] == 8:
        return {"p": s["p"], "m": s["m"].view(torch.float8_e4m3fn), "m step": s["m_scale"], "v codes": s["v"], "v step": s["v_scale"]}
    return {"p": s["p"], "m": s["m"], "v": s["v"]}


# ----------------------------------------------------------------- in plain torch operations
def _words(n, seed, tensor_id, device):
    """Philox4x32-10 words of the flat indices 0 .. n - 1 of a tensor."""
    low = 0xFFFFFFFF
    j = torch.arange((n + 3) // 4, dtype=torch.int64, device=device)
    c0, c1, c2, c3 = j & low, j >> 32, torch.full_like(j, tensor_id & low), torch.full_like(j, tensor_id >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], 1).view(-1)[:n]


def _code(x, u, top, shift):
    """8-bit codes of x (a whole number of 128-blocks) and step sizes: |x| / step is cut to the grid's mantissa after adding the
    threshold u in [0, 2^16), so that it goes up with the probability of what is cut off.  shift = 20: sign and E4M3, 19: E4M4."""
    x = x.view(-1, BLK)
    amax = x.abs().amax(1, keepdim=True)
    q = top / amax.double()
    inv = q.float()
    inv = torch.where(inv.double() > q, torch.nextafter(inv, torch.zeros_like(inv)), inv)      # rounded toward zero
    dead = (amax == 0) | torch.isinf(top / amax)
    inv, step = torch.where(dead, 0.0, inv), torch.where(dead, 0.0, amax / top)
    # times 2^-120 the grid's exponents are binary32's own, subnormal numbers included
    bits = (x.abs() * inv * 2.0 ** -120).view(torch.int32).long()
    codes = (bits + (u.view(-1, BLK) << (shift - 16)) + (1 << (shift - 17))) >> shift
    if shift == 19:
        codes = torch.where((x > 0) & ~dead, codes.clamp(min=1), codes)       # a second moment that is not zero stays so
    else:
        codes = codes | torch.where(x < 0, 128, 0)
    return codes.to(torch.uint8).view(-1), step.view(-1)


def _decode_v(codes, step):
    c = codes.int()
    return ((c << 19).view(torch.float32) * 2.0 ** 120) * step.repeat_interleave(BLK)


def _plain_adamw(s):
    case, h = s["case"], ADAMW
    sizes, starts = _flat(case)
    lo, hi = None, None
    if case["bits"] == 8 or case["dtype"] == "bf16":
        word = torch.zeros(starts[-1], dtype=torch.int64, device=s["p"].device)
        for i, (n, a) in enumerate(zip(sizes, starts)):
            word[a:a + n] = _words(n, SEED, TENSOR_ID + i + (h["step"] << 32), s["p"].device)
        lo, hi = word & 0xFFFF, word >> 16
        del word
    p, g = s["p"].float(), s["g"].float()
    if case["bits"] == 8:
        m = s["m"].view(torch.float8_e4m3fn).float() * s["m_scale"].repeat_interleave(BLK)
        v = _decode_v(s["v"], s["v_scale"])
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1.0 - h["beta2"])
    del g
    b1, b2 = 1.0 - h["beta1"] ** h["step"], 1.0 - h["beta2"] ** h["step"]
    p = p * (1.0 - h["lr"] * h["weight_decay"]) - (h["lr"] / b1) * (m / (torch.sqrt(v) / math.sqrt(b2) + h["eps"]))
    if case["dtype"] == "bf16":                # sixteen bits are cut off, after a threshold of sixteen bits was added
        p = (((p.view(torch.int32).long() + lo) >> 16) << 16).to(torch.int32).view(torch.float32)
    s["p"].copy_(p)
    del p
    if case["bits"] == 8:
        for name, x, u, top, shift in (("m", m, lo ^ hi, M_MAX, 20), ("v", v, hi, V_MAX, 19)):
            codes, step = _code(x, u, top, shift)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(step)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _moments(s)


def _softmax(x):
    """(shifted logits, their exponentials, sum of these) in 32 bits."""
    z = x - x.amax(1, keepdim=True)
    e = torch.exp(z)
    return z, e, e.sum(1, keepdim=True)


def _plain_gradient(e, total, targets, c, dtype):
    """c ([j = target] - p_j) from the exponentials, which it overwrites."""
    d = e.div_(total).mul_(-c[:, None])
    d.scatter_add_(1, targets[:, None], c[:, None])
    return d.to(_dtype(dtype))


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        out = s["table"].float()[s["ids"].clamp(min=0)] * case["scale"]
        return {"out": torch.where(s["ids"][:, None] >= 0, out, 0.0).to(_dtype(case["dtype"]))}
    if op == "embed_bwd":
        ids, order = torch.sort(s["ids"], stable=True)
        first = int(case["t"] // 20)           # padding sorts to the front
        rows = s["dout"].float()[order[first:]].double()
        out = torch.zeros(case["v"], case["d"], dtype=torch.float64, device=rows.device).index_add_(0, ids[first:], rows)
        return {"dtable": (out * case["scale"]).float()}
    if op == "adamw":
        return _plain_adamw(s)
    targets = s["targets"]
    z, e, total = _softmax(s["logits"].float())
    logp = z.gather(1, targets[:, None])[:, 0] - torch.log(total[:, 0])
    del z
    if op == "policy":
        w, a = s["weight"], s["advantage"]
        use = w != 0
        logp = torch.where(use, logp, 0.0)
        rho = torch.exp(logp - s["old"])
        plain, clipped = rho * a, rho.clamp(1.0 - CLIP, 1.0 + CLIP) * a
        row = -torch.minimum(plain, clipped)
        c = torch.where(plain <= clipped, -plain, 0.0)
        if s["ref"] is not None:
            k = torch.exp(s["ref"] - logp)
            row, c = row + KL_COEF * (k - (s["ref"] - logp) - 1.0), c + KL_COEF * (1.0 - k)
        row, c = torch.where(use, w * row, 0.0), torch.where(use, w * c, 0.0)
        return {"loss": row.double().sum().float().view(1), "row_loss": row, "logp": logp, "dlogits": _plain_gradient(e, total, targets, c, case["dtype"])}
    n = s["offsets"][1:] - s["offsets"][:-1]
    side = torch.repeat_interleave(torch.arange(2 * case["pairs"], device=n.device), n)
    ratio = torch.zeros(2 * case["pairs"], dtype=torch.float64, device=n.device).index_add_(0, side, (logp - s["ref"]).double()).view(-1, 2)
    h = (BETA * (ratio[:, 0] - ratio[:, 1])).float()
    pair = (1.0 - SMOOTHING) * torch.log1p(torch.exp(-h)) + SMOOTHING * torch.log1p(torch.exp(h))
    dh = (SMOOTHING - 1.0 / (1.0 + torch.exp(h))) * (BETA / case["pairs"])      # the same as -(1 - e) sigma(-h) + e sigma(h)
    c = torch.stack([dh, -dh], 1).view(-1)[side]
    return {"loss": pair.double().mean().float().view(1), "pair_loss": pair, "logp": logp, "dlogits": _plain_gradient(e, total, targets, c, case["dtype"])}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_e4m4(codes):
    """Numbers of the second moment's codes: four bits of exponent, four of mantissa, no sign."""
    c = codes.long()
    e, m = c // 16, (c % 16).double()
    return torch.where(e == 0, m / 1024.0, (16.0 + m) * torch.exp2(e.double() - 11.0))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        keep = (s["ids"] >= 0).double()[:, None]
        return {"out": case["scale"] * torch.index_select(s["table"], 0, s["ids"].relu()).double() * keep}
    if op == "embed_bwd":
        out = torch.zeros((case["v"] + 1, case["d"]), dtype=torch.float64, device="cuda")
        where = torch.where(s["ids"] < 0, case["v"], s["ids"])
        out.scatter_add_(0, where[:, None].expand(-1, case["d"]), s["dout"].double())
        return {"dtable": case["scale"] * out[:-1]}
    if op == "adamw":
        h = ADAMW
        m, v, g, p = s["m"], s["v"], s["g"].double(), s["p"].double()
        coded = case["bits"] == 8
        spread = lambda name: s[name].double().view(-1, 1).expand(-1, BLK).reshape(-1)  # noqa: E731
        m = m.view(torch.float8_e4m3fn).double() * spread("m_scale") if coded else m.double()
        v = _exact_e4m4(v) * spread("v_scale") if coded else v.double()
        m += (1.0 - h["beta1"]) * (g - m)
        v += (1.0 - h["beta2"]) * (g ** 2 - v)
        del g
        out = {}
        if coded:
            for name, x, top in (("m", m, M_MAX), ("v", v, V_MAX)):
                big = x.view(-1, BLK).abs().max(1).values
                out[name + " step"] = big / top
                if name == "m":
                    out[name] = (x.view(-1, BLK) / torch.where(big > 0, big / top, 1.0)[:, None]).view(-1)
            out["v codes"] = None
        else:
            out = {"m": m, "v": v}
        mean = m / -math.expm1(h["step"] * math.log(h["beta1"]))
        root = (v / -math.expm1(h["step"] * math.log(h["beta2"]))) ** 0.5
        out["p"] = p - h["lr"] * (h["weight_decay"] * p + mean / (root + h["eps"]))
        return out
    x, target = s["logits"].double(), s["targets"][:, None]
    lse = torch.logsumexp(x, 1)
    logp = torch.take_along_dim(x, target, 1)[:, 0] - lse
    if op == "policy":
        w, a, logp = s["weight"].double(), s["advantage"].double(), torch.where(s["weight"] == 0, torch.zeros_like(logp), logp)
        ratio = (logp - s["old"].double()).exp()
        gain = torch.where(a >= 0, ratio.clamp(max=1.0 + CLIP), ratio.clamp(min=1.0 - CLIP)) * a
        inside = torch.where(a >= 0, ratio <= 1.0 + CLIP, ratio >= 1.0 - CLIP)
        row, slope = -gain, -(ratio * a) * inside
        if s["ref"] is not None:
            d = s["ref"].double() - logp
            row += KL_COEF * (d.expm1() - d)
            slope -= KL_COEF * d.expm1()
        row, slope = w * row, w * slope
        out = {"loss": row.sum().view(1), "row_loss": row, "logp": logp}
    else:
        ends = s["offsets"].tolist()
        diff = logp - s["ref"].double()
        sums = torch.stack([diff[i:j].sum() for i, j in zip(ends, ends[1:])])
        h = BETA * (sums[0::2] - sums[1::2])
        up, down = torch.nn.functional.logsigmoid(h), torch.nn.functional.logsigmoid(-h)
        pair = -(1.0 - SMOOTHING) * up - SMOOTHING * down
        dh = (-(1.0 - SMOOTHING) * torch.sigmoid(-h) + SMOOTHING * torch.sigmoid(h)) * BETA / len(h)
        slope = torch.empty_like(logp)
        for k, (i, j) in enumerate(zip(ends, ends[1:])):
            slope[i:j] = dh[k // 2] if k % 2 == 0 else -dh[k // 2]
        out = {"loss": pair.mean().view(1), "pair_loss": pair, "logp": logp}
    p = x.sub_(lse[:, None]).exp_()
    p.mul_(-slope[:, None])
    p.scatter_add_(1, target, slope[:, None])
    out["dlogits"] = p
    return out
