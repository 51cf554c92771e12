"""The block-scaled 8-bit operators of a transformer layer, as they are measured.

Five operators around the quantized linear layer, all on E4M3 codes with one binary32 step size for
every block of 128 values along the contracted axis (1 x 128), or for every 128 x 128 tile:

  quantize   x -> codes and step sizes, row-major and / or transposed; x is binary32, bfloat16 or
             itself a matrix of block codes (an 8-bit activation checkpoint on its way into the
             weight gradient, whose contraction runs over the tokens)
  product    out = A B^T over block codes
  norm       r = x + residual, y = r / rms(r) * w, y leaves as block codes; and its backward pass
  glu        h = act(X Wg^T) * (X Wu^T), h leaves as block codes, gate and up projections as 8-bit
             checkpoints; and its backward pass, which reads the checkpoints

`run` computes a case in plain 32-bit torch operations where `own` is false, and through the
library where it is true.  `exact` computes it from the definitions in 64 bits.
"""
import math

import torch

own = False

BLK = 128
E4M3_MAX = 448.0
EPS = 1e-5


def listed():
    return [
        # one generated token through a 4096-wide projection: reading the weights is all there is
        {"name": "product token", "op": "product", "m": 1, "n": 4096, "k": 4096, "b_tile": True, "out": "bf16"},
        # a handful of prompts, a ragged batch, through the fused query/key/value projection (2048 -> 2560)
        {"name": "product ragged batch", "op": "product", "m": 333, "n": 2560, "k": 2048, "b_tile": True, "out": "bf16"},
        # the forward product of a training step on a 4096 x 4096 layer
        {"name": "product train", "op": "product", "m": 16384, "n": 4096, "k": 4096, "b_tile": True, "out": "bf16"},
        # a weight gradient of the 2048 -> 5632 projection: contraction over 8192 tokens, both operands in 1 x 128 blocks
        {"name": "product weight gradient", "op": "product", "m": 5632, "n": 2048, "k": 8192, "b_tile": False, "out": "f32"},
        # the norm before a projection, one generated token
        {"name": "norm token", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "residual": True},
        # the norm of a training step
        {"name": "norm train", "op": "norm", "rows": 16384, "cols": 4096, "dtype": "bf16", "residual": True},
        # its backward pass in binary32 on 2048 features, an odd number of tokens
        {"name": "norm backward", "op": "norm_bwd", "rows": 8191, "cols": 2048, "dtype": "f32", "residual": True},
        # four sequences generating a token each through the gated block 2048 -> 5632
        {"name": "glu tokens", "op": "glu", "t": 4, "f": 5632, "k": 2048, "act": "silu", "checkpoint": False},
        # the gated block of a training step, with the checkpoints for its backward pass
        {"name": "glu train", "op": "glu", "t": 16384, "f": 5632, "k": 2048, "act": "silu", "checkpoint": True},
        # its backward pass: gradients of both projections in both layouts and h^T for the weight gradient after it
        {"name": "glu backward", "op": "glu_bwd", "t": 16384, "f": 5632, "act": "silu", "dtype": "bf16"},
        # weights once per step: 128 x 128 tiles in both layouts
        {"name": "quantize weights", "op": "quantize", "rows": 5632, "cols": 2048, "dtype": "f32", "tile": True, "rm": True, "tr": True},
        # an 8-bit activation checkpoint turned over for the weight gradient
        {"name": "quantize checkpoint", "op": "quantize", "rows": 16384, "cols": 2048, "dtype": "e4m3", "tile": False, "rm": False, "tr": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["product", "product", "norm", "norm_bwd", "glu", "glu", "glu_bwd", "quantize"])
    if op == "product":
        if rng.random() < 0.25:      # weight gradients: the contraction runs over the tokens
            return {"op": op, "m": _log(rng, 256, 5632), "n": _log(rng, 256, 4096), "k": _log(rng, 128, 8192),
                    "b_tile": rng.random() < 0.5, "out": "f32"}
        return {"op": op, "m": _log(rng, 1, 16384), "n": _log(rng, 128, 4096), "k": _log(rng, 128, 4096),
                "b_tile": rng.random() < 0.8, "out": rng.choice(["bf16", "bf16", "f32"])}
    if op in ("norm", "norm_bwd"):
        return {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 128, 4096), "dtype": rng.choice(["bf16", "f32"]),
                "residual": rng.random() < 0.75}
    if op == "glu":
        return {"op": op, "t": _log(rng, 1, 16384), "f": _log(rng, 128, 5632), "k": _log(rng, 128, 2048),
                "act": rng.choice(["silu", "gelu"]), "checkpoint": rng.random() < 0.5}
    if op == "glu_bwd":
        return {"op": op, "t": _log(rng, 1, 16384), "f": _log(rng, 128, 5632), "act": rng.choice(["silu", "gelu"]),
                "dtype": rng.choice(["bf16", "f32"])}
    rm = rng.random() < 0.7
    return {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 128, 4096), "dtype": rng.choice(["f32", "bf16", "e4m3"]),
            "tile": rng.random() < 0.5, "rm": rm, "tr": (not rm) or rng.random() < 0.7}


def _blocks(n):
    return (n + BLK - 1) // BLK


def work(case):
    """Bytes: every input and output once.  Flops: the products' multiply-adds."""
    op = case["op"]
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        sb = _blocks(n) if case["b_tile"] else n
        return {"bytes": (m + n) * k + 4 * (m + sb) * _blocks(k) + m * n * (2 if case["out"] == "bf16" else 4), "flops": 2 * m * n * k}
    if op == "norm":
        r, c, e = case["rows"], case["cols"], 2 if case["dtype"] == "bf16" else 4
        moved = r * c * (e + 1 + (2 * e if case["residual"] else 0))
        return {"bytes": moved + c * e + 4 * r * (_blocks(c) + 1), "flops": 6 * r * c}
    if op == "norm_bwd":
        r, c, e = case["rows"], case["cols"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": r * c * e * (4 if case["residual"] else 3) + c * (e + 4) + 4 * r, "flops": 9 * r * c}
    if op == "glu":
        t, f, k = case["t"], case["f"], case["k"]
        out = t * f + 4 * t * _blocks(f)
        return {"bytes": (t + 2 * f) * k + 4 * (t + 2 * _blocks(f)) * _blocks(k) + out * (3 if case["checkpoint"] else 1), "flops": 4 * t * f * k}
    if op == "glu_bwd":
        t, f = case["t"], case["f"]
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": t * f * (e + 2 + 5) + 4 * (4 * t * _blocks(f) + 3 * f * _blocks(t)), "flops": 20 * t * f}
    r, c = case["rows"], case["cols"]
    e = {"f32": 4, "bf16": 2, "e4m3": 1}[case["dtype"]]
    n = int(case["rm"]) + int(case["tr"])
    return {"bytes": r * c * (e + n) + 4 * r * c * (n + (case["dtype"] == "e4m3")) // BLK, "flops": 3 * r * c}


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _randn(g, *shape, std=1.0):
    x = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)
    return x.mul_(std) if std != 1.0 else x


def _features(g, rows, cols):
    """Activations as a network has them: a few feature columns much larger than the rest, tokens of different size."""
    return _randn(g, rows, cols) * torch.exp(0.8 * _randn(g, 1, cols)) * torch.exp(0.3 * _randn(g, rows, 1))


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _pad(n, m):
    return (n + m - 1) // m * m


def _empty_blocks(rows, cols, tile=False):
    """Codes with a pitch of a multiple of 16 bytes, step sizes with a pitch of a multiple of 4."""
    codes = torch.zeros((rows, _pad(cols, 16)), dtype=torch.uint8, device="cuda")[:, :cols]
    scale = torch.zeros((_blocks(rows) if tile else rows, _pad(_blocks(cols), 4)), device="cuda")[:, :_blocks(cols)]
    return codes, scale, BLK if tile else 1


def _coded(x, tile=False):
    """Block codes of x: what an earlier step of the program left behind."""
    codes, scale, rows = _empty_blocks(*x.shape, tile)
    c, s = _plain_quantize(x, tile)
    codes.copy_(c.view(torch.uint8))
    scale.copy_(s)
    return codes, scale, rows


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], {"case": case}
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _coded(_features(g, m, k))
        s["b"] = _coded(_randn(g, n, k, std=0.02), True) if case["b_tile"] else _coded(_features(g, n, k))
        s["out"] = torch.empty((m, n), dtype=_dtype(case["out"]), device="cuda")
    elif op in ("norm", "norm_bwd"):
        r, c, dt = case["rows"], case["cols"], _dtype(case["dtype"])
        s["x"] = _features(g, r, c).to(dt)
        s["residual"] = _features(g, r, c).to(dt) if case["residual"] else None
        s["w"] = (1.0 + 0.2 * _randn(g, c)).to(dt)
        s["rstd"] = torch.empty(r, device="cuda")
        if op == "norm":
            s["r"] = torch.empty((r, c), dtype=dt, device="cuda") if case["residual"] else None
            s["y"] = _empty_blocks(r, c)
        else:
            s["dy"] = _randn(g, r, c, std=1e-2).to(dt)
            s["rstd"].copy_(torch.rsqrt(s["x"].float().square().mean(1) + EPS))
            s["dx"] = torch.empty((r, c), dtype=dt, device="cuda")
            s["dw"] = torch.empty(c, device="cuda")
            # partial sums of the weight's gradient: 512 rows of them suffice for any input
            s["ws"] = torch.empty(4 * 512 * _pad(c, 64), dtype=torch.uint8, device="cuda")
    elif op == "glu":
        t, f, k = case["t"], case["f"], case["k"]
        s["x"] = _coded(_randn(g, t, k))
        s["wg"], s["wu"] = _coded(_randn(g, f, k, std=k ** -0.5), True), _coded(_randn(g, f, k, std=k ** -0.5), True)
        s["h"] = _empty_blocks(t, f)
        s["gate"], s["up"] = (_empty_blocks(t, f), _empty_blocks(t, f)) if case["checkpoint"] else (None, None)
    elif op == "glu_bwd":
        t, f = case["t"], case["f"]
        s["gate"], s["up"] = _coded(_randn(g, t, f)), _coded(_randn(g, t, f))
        s["dh"] = (1e-3 * _features(g, t, f)).to(_dtype(case["dtype"]))
        s["dg"], s["du"] = _empty_blocks(t, f), _empty_blocks(t, f)
        s["dg_t"], s["du_t"], s["h_t"] = _empty_blocks(f, t), _empty_blocks(f, t), _empty_blocks(f, t)
    else:
        r, c = case["rows"], case["cols"]
        x = _features(g, r, c)
        s["x"] = _coded(x) if case["dtype"] == "e4m3" else x.to(_dtype(case["dtype"]))
        s["rm"] = _empty_blocks(r, c, case["tile"]) if case["rm"] else None
        s["tr"] = _empty_blocks(c, r, case["tile"]) if case["tr"] else None
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _answers(matrices):
    """Block-coded matrices as the E4M3 numbers they hold and their step sizes."""
    return {**{n: b[0].view(torch.float8_e4m3fn) for n, b in matrices.items()}, **{n + " step": b[1] for n, b in matrices.items()}}


# ----------------------------------------------------------------- in the framework
def _run_own(s):
    import paper_2511_00874_b200 as srq
    case = s["case"]
    op = case["op"]
    b = lambda name: None if s[name] is None else srq.Blocks(*s[name])  # noqa: E731
    act = {"silu": srq.SILU, "gelu": srq.GELU}.get(case.get("act"))
    if op == "product":
        srq.srq_gemm_blocks(b("a"), b("b"), s["out"], device_status=s["status"])
        return {"out": s["out"]}
    if op == "norm":
        srq.srq_rmsnorm_fwd(s["x"], s["residual"], s["w"], EPS, b("y"), s["r"], s["rstd"], device_status=s["status"])
        return {**_answers({"y": s["y"]}), "rstd": s["rstd"], "r": s["r"]}
    if op == "norm_bwd":
        srq.srq_rmsnorm_bwd(s["dy"], s["x"], s["w"], s["rstd"], s["residual"], s["dx"], s["dw"], ws=s["ws"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if op == "glu":
        srq.srq_glu_fwd(b("x"), b("wg"), b("wu"), act, b("h"), b("gate"), b("up"), device_status=s["status"])
        names = ("h", "gate", "up") if case["checkpoint"] else ("h",)
    elif op == "glu_bwd":
        srq.srq_glu_bwd(s["dh"], b("gate"), b("up"), act, srq.BLOCK_RNE, b("dg"), b("du"), b("dg_t"), b("du_t"), b("h_t"),
                        device_status=s["status"])
        names = ("dg", "du", "dg_t", "du_t", "h_t")
    else:
        x = srq.Blocks(*s["x"]) if case["dtype"] == "e4m3" else s["x"]
        srq.srq_quantize_blocks(x, srq.BLOCK_RNE, b("rm"), b("tr"), device_status=s["status"])
        names = tuple(n for n in ("rm", "tr") if case[n])
    return _answers({n: s[n] for n in names})


# ----------------------------------------------------------------- in plain torch operations
def _plain_steps(amax):
    """Step size amax / 448 and its reciprocal, 448 / amax rounded toward zero."""
    q = E4M3_MAX / amax.double()
    inv = q.float()
    inv = torch.where(inv.double() > q, torch.nextafter(inv, torch.zeros_like(inv)), inv)
    dead = (amax == 0) | torch.isinf(E4M3_MAX / amax)
    zero = torch.zeros_like(inv)
    return torch.where(dead, zero, amax / E4M3_MAX), torch.where(dead, zero, inv)


def _plain_quantize(x, tile=False):
    """(codes, step sizes) of 1 x 128 blocks or 128 x 128 tiles of a 32-bit x."""
    r, c = x.shape
    nb, br = _blocks(c), BLK if tile else 1
    full = torch.nn.functional.pad(x, (0, nb * BLK - c, 0, _pad(r, br) - r))
    full = full.view(-1, br, nb, BLK)
    step, inv = _plain_steps(full.abs().amax(dim=(1, 3)))
    codes = (full * inv[:, None, :, None]).to(torch.float8_e4m3fn)
    return codes.view(-1, nb * BLK)[:r, :c], step


def _plain_values(blocks):
    codes, scale, rows = blocks
    r, c = codes.shape
    v = codes.view(torch.float8_e4m3fn).float()
    s = scale.repeat_interleave(rows, 0)[:r] if rows > 1 else scale
    return v * s.repeat_interleave(BLK, 1)[:, :c]


def _plain_act(g, act):
    """act(g) and act'(g)."""
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "product":
        return {"out": (_plain_values(s["a"]) @ _plain_values(s["b"]).t()).to(_dtype(case["out"]))}
    if op == "norm":
        r = s["x"].float()
        if case["residual"]:
            r = r + s["residual"].float()
        rstd = 1.0 / torch.sqrt((r * r).mean(1) + EPS)
        y = _plain_quantize(r * rstd[:, None] * s["w"].float())
        return {**_answers({"y": y}), "rstd": rstd, "r": r.to(s["x"].dtype) if case["residual"] else None}
    if op == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = s["x"].float() * rstd
        wdy = dy * s["w"].float()
        dx = rstd * (wdy - xhat * (wdy * xhat).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(s["x"].dtype), "dw": (dy * xhat).sum(0)}
    if op == "glu":
        x = _plain_values(s["x"])
        gate, up = x @ _plain_values(s["wg"]).t(), x @ _plain_values(s["wu"]).t()
        h = _plain_act(gate, case["act"])[0] * up
        values = {"h": h, "gate": gate, "up": up} if case["checkpoint"] else {"h": h}
        return _answers({n: _plain_quantize(v) for n, v in values.items()})
    if op == "glu_bwd":
        gate, up, dh = _plain_values(s["gate"]), _plain_values(s["up"]), s["dh"].float()
        a, da = _plain_act(gate, case["act"])
        dg, du, h = dh * up * da, dh * a, a * up
        values = {"dg": dg, "du": du, "dg_t": dg.t(), "du_t": du.t(), "h_t": h.t()}
        return _answers({n: _plain_quantize(v) for n, v in values.items()})
    x = _plain_values(s["x"]) if case["dtype"] == "e4m3" else s["x"].float()
    values = {n: x if n == "rm" else x.t() for n in ("rm", "tr") if case[n]}
    return _answers({n: _plain_quantize(v, case["tile"]) for n, v in values.items()})


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_numbers(blocks):
    """The numbers a block-coded matrix stands for."""
    codes, scale, rows = blocks
    n, m = codes.shape
    number = codes.contiguous().view(torch.float8_e4m3fn).double()
    i = torch.arange(n, device="cuda") // rows
    j = torch.arange(m, device="cuda") // BLK
    return number.mul_(scale.double()[i][:, j])


def _exact_blocks(name, v, rows=1):
    """Quotients v / D before their rounding to 8 bits, and the step sizes D = max |v| / 448."""
    n, m = v.shape
    i, j = torch.arange(n, device="cuda") // rows, torch.arange(m, device="cuda") // BLK
    big = torch.zeros((-(-n // rows), -(-m // BLK)), dtype=torch.float64, device="cuda")
    by_row = torch.zeros((n, big.shape[1]), dtype=torch.float64, device="cuda").index_reduce_(1, j, v.abs(), "amax")
    step = big.index_reduce_(0, i, by_row, "amax") / E4M3_MAX
    return {name: v / torch.where(step > 0, step, 1.0)[i][:, j], name + " step": step}


def _exact_gate(g, act):
    if act == "silu":
        p = torch.sigmoid(g)
        return p * g, p + g * p * torch.sigmoid(-g)
    k = (2.0 / math.pi) ** 0.5
    u = k * g + (k * 0.044715) * g ** 3
    p = torch.sigmoid(2.0 * u)             # (1 + tanh u) / 2
    return g * p, p + g * 2.0 * p * torch.sigmoid(-2.0 * u) * (k + (3.0 * k * 0.044715) * g ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        return {"out": torch.einsum("mk,nk->mn", _exact_numbers(s["a"]), _exact_numbers(s["b"]))}
    if op == "norm":
        r = s["x"].double()
        if s["residual"] is not None:
            r += s["residual"].double()
        rms = (r.square().sum(1) / r.shape[1] + EPS).sqrt()
        out = _exact_blocks("y", r / rms[:, None] * s["w"].double())
        return {**out, "rstd": rms.reciprocal(), "r": r if s["residual"] is not None else None}
    if op == "norm_bwd":
        n = s["x"].double() * s["rstd"].double()[:, None]
        gy = s["dy"].double()
        gn = gy * s["w"].double()
        dx = (gn - n * ((gn * n).sum(1) / n.shape[1])[:, None]) * s["rstd"].double()[:, None]
        if s["residual"] is not None:
            dx += s["residual"].double()
        return {"dx": dx, "dw": torch.einsum("rc,rc->c", gy, n)}
    if op == "glu":
        x = _exact_numbers(s["x"])
        g = torch.einsum("tk,fk->tf", x, _exact_numbers(s["wg"]))
        u = torch.einsum("tk,fk->tf", x, _exact_numbers(s["wu"]))
        out = _exact_blocks("h", _exact_gate(g, case["act"])[0] * u)
        if case["checkpoint"]:
            out.update(_exact_blocks("gate", g))
            out.update(_exact_blocks("up", u))
        return out
    if op == "glu_bwd":
        g, u, dh = _exact_numbers(s["gate"]), _exact_numbers(s["up"]), s["dh"].double()
        a, slope = _exact_gate(g, case["act"])
        out = _exact_blocks("h_t", (a * u).t().contiguous())
        dg, du = dh * u * slope, dh * a
        del a, slope, g, u, dh
        for name, v in (("dg", dg), ("du", du)):
            out.update(_exact_blocks(name, v))
            out.update(_exact_blocks(name + "_t", v.t().contiguous()))
        return out
    x = _exact_numbers(s["x"]) if case["dtype"] == "e4m3" else s["x"].double()
    rows, out = BLK if case["tile"] else 1, {}
    if case["rm"]:
        out.update(_exact_blocks("rm", x, rows))
    if case["tr"]:
        out.update(_exact_blocks("tr", x.t().contiguous(), rows))
    return out
