"""Microscaled (MX) 4- and 8-bit operators, as cases that can be timed and compared with their plain form.

What a calibrated rotation is for: activations and weights that it has freed of outliers are stored in blocks of 32 values with one
power of two as their scale, and multiplied in that form.  A case's "op" says which operator one pass runs:

* ``norm``       the residual's addition and the RMS norm of token rows, its result in MX blocks, read back as values.
* ``quantize``   a matrix (activations, weights) into MX blocks, read back as values.
* ``objective``  the calibration objective that belongs to them: squared error of the MX quantiser on a rotated block, and its gradient.
* ``product``    C = A B^T of two MX matrices, as a linear layer runs it on token rows.

Formats: "mxfp4" holds 4-bit floats of 1 sign, 2 exponent and 1 mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), "mxfp8" 8-bit floats of 1, 4
and 3 bits (largest 448).  Of a block with largest magnitude a, the scale is 2^E, E = max(floor(log2 a) - e, -127) with e = 2 or 8, and
every value v becomes 2^E times the representable value nearest to v / 2^E, ties to the even code, never beyond the largest.

Stored form, as the library takes it: two 4-bit codes a byte, the lower nibble first, or one 8-bit code a byte; E + 127 in a byte a block;
a row's codes are filled up with zeros to whole blocks, its scales to a multiple of 16 bytes.
"""

import functools
import math

import torch

own = False

_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_EMAX = {"mxfp4": 2, "mxfp8": 8}
_TOP = {"mxfp4": 6.0, "mxfp8": 448.0}
_EPS = 1e-5


def listed():
    def norm(name, tokens, n, x, fmt, residual=True, gain=False):
        return {"name": name, "op": "norm", "tokens": tokens, "n": n, "x": x, "format": fmt, "residual": residual, "gain": gain}

    def quantize(name, tokens, n, x, fmt):
        return {"name": name, "op": "quantize", "tokens": tokens, "n": n, "x": x, "format": fmt}

    def objective(name, b, tokens, n, grad, fmt, reduce):
        return {"name": name, "op": "objective", "b": b, "tokens": tokens, "n": n, "grad": grad, "format": fmt, "reduce": reduce}

    def product(name, m, n, k, a, b, out):
        return {"name": name, "op": "product", "m": m, "n": n, "k": k, "a": a, "b": b, "out": out}

    return [
        # one token of a model with rotated residual stream on its way into a linear layer: latency alone
        norm("norm_token", 1, 4096, "bf16", "mxfp4"),
        # a prompt of a model whose norm keeps its gain, 8-bit activations
        norm("norm_prompt", 8192, 4096, "bf16", "mxfp8", gain=True),
        # fp32 rows whose last block is cut short
        norm("norm_ragged", 1023, 5004, "f32", "mxfp4"),
        # a block of activations behind a rotation, at a pruned width
        quantize("quantize_ragged", 333, 2890, "f32", "mxfp8"),
        # the weights of a large layer, once a model
        quantize("quantize_weights", 8192, 8192, "bf16", "mxfp4"),
        # the calibration's rotated block at its ordinary size
        objective("objective_block", 1, 8192, 4096, "bf16", "mxfp4", "mean"),
        # every head of a layer in one call
        objective("objective_heads", 64, 2048, 128, "f32", "mxfp8", "sum"),
        # single-token serving: reads the weights once
        product("product_token", 1, 4096, 4096, "mxfp4", "mxfp4", "bf16"),
        # a few users' tokens against 4-bit weights
        product("product_users", 24, 8192, 4096, "mxfp8", "mxfp4", "bf16"),
        # a short prompt, at sizes that are multiples of nothing
        product("product_ragged", 515, 2890, 5100, "mxfp4", "mxfp4", "f32"),
        # prompts at the two model sizes that the benchmark is quoted on
        product("product_prompt", 8192, 4096, 4096, "mxfp4", "mxfp4", "bf16"),
        product("product_large", 8192, 8192, 8192, "mxfp8", "mxfp8", "bf16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Widths from a small head's to the largest rotation's, one token to a long prompt, mostly odd sizes."""
    op = rng.choice(["norm", "quantize", "objective", "product"])
    fmt = rng.choice(["mxfp4", "mxfp8"])
    if op == "product":
        return {"op": op, "m": _spread(rng, 1, 8192), "n": _spread(rng, 64, 8192), "k": _spread(rng, 64, 8192), "a": fmt,
                "b": rng.choice(["mxfp4", "mxfp8"]), "out": rng.choice(["bf16", "f32"])}
    if op == "objective":
        b = _spread(rng, 1, 64)
        n = _spread(rng, 64, 8192 // b) if b < 64 else _spread(rng, 64, 128)
        return {"op": op, "b": b, "tokens": _spread(rng, 16, max(32, min(8192, 2 ** 25 // (b * n)))), "n": n, "grad": rng.choice(["bf16", "f32"]),
                "format": fmt, "reduce": rng.choice(["mean", "sum"])}
    case = {"op": op, "tokens": _spread(rng, 1, 8192), "n": _spread(rng, 64, 8192), "x": rng.choice(["bf16", "f32"]), "format": fmt}
    if op == "norm":
        case["residual"] = rng.random() < 0.75
        case["gain"] = rng.random() < 0.5
    return case


# ---- data

def _up(x, m):
    return -(-x // m) * m


def _rows(shape, dtype, generator=None, values=None):
    """A matrix (or a stack of them) whose rows start at multiples of eight elements, as the library wants them."""
    *lead, n = shape
    buf = torch.empty((*lead, _up(n, 8)), dtype=dtype, device="cuda")
    if values is not None:
        buf[..., :n] = values
    return buf[..., :n]


def _activations(shape, g):
    """Rows behind a rotation: near normal, each token at a level of its own, a few channels still above the others."""
    x = torch.randn(shape, device="cuda", generator=g)
    level = torch.exp(0.5 * torch.randn((*shape[:-1], 1), device="cuda", generator=g))
    channel = 1.0 + 3.0 * (torch.rand((shape[-1],), device="cuda", generator=g) > 0.995).float()
    return x * level * channel


def _code_buffers(rows, n, fmt):
    nb = _up(n, 32) // 32
    codes = torch.empty((rows, nb * (16 if fmt == "mxfp4" else 32)), dtype=torch.uint8, device="cuda")
    return codes, torch.empty((rows, _up(nb, 16)), dtype=torch.uint8, device="cuda")


def _stored(values, fmt):
    """Codes and scales of a matrix in the stored form."""
    rows, n = values.shape
    codes, scales = _code_buffers(rows, n, fmt)
    level, exponent = _to_blocks(values, fmt)
    if fmt == "mxfp4":
        code = torch.bucketize(level.abs(), _levels4()[:8]).to(torch.uint8) | (torch.signbit(level).to(torch.uint8) << 3)
        code = code.reshape(rows, -1, 2)
        codes.copy_(code[..., 0] | (code[..., 1] << 4))
    else:
        codes.copy_(level.to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, -1))
    scales.zero_()
    scales[:, :exponent.shape[1]] = (exponent + 127).to(torch.uint8).squeeze(-1)
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["A"], s["As"] = _stored(_activations((m, k), g), case["a"])
        s["B"], s["Bs"] = _stored(torch.randn((n, k), device="cuda", generator=g) / math.sqrt(k), case["b"])
        s["C"] = _rows((m, n), _TYPE[case["out"]])
        return s
    if op == "objective":
        shape = (case["b"], case["tokens"], case["n"])
        s["Y"] = _rows(shape, torch.float32, values=_activations(shape, g))
        s["dY"] = _rows(shape, _TYPE[case["grad"]])
        s["loss"] = torch.empty(case["b"], device="cuda")
        return s
    shape = (case["tokens"], case["n"])
    dtype = _TYPE[case["x"]]
    s["X"] = _rows(shape, dtype, values=_activations(shape, g))
    s["codes"], s["scales"] = _code_buffers(*shape, case["format"])
    s["values"] = _rows(shape, dtype)
    if op == "norm":
        s["R"] = _rows(shape, dtype, values=4.0 * _activations(shape, g)) if case["residual"] else None
        s["H"] = _rows(shape, dtype) if case["residual"] else None
        s["g"] = 1.0 + 0.2 * torch.randn(case["n"], device="cuda", generator=g) if case["gain"] else None
    return s


# ---- plain form

@functools.lru_cache(None)
def _powers():
    return torch.tensor([math.ldexp(1.0, i - 127) for i in range(255)], device="cuda")


@functools.lru_cache(None)
def _levels4():
    positive = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    return torch.cat((positive, -positive))


def _power(e):
    """2^e for integers -127 <= e <= 127, exactly (torch.ldexp takes a pow, which is off by a rounding for some)."""
    return _powers()[e + 127]


def _to_blocks(values, fmt):
    """(levels, exponents) of rows of fp32 values: blocks of 32 whose values stand for level * 2^exponent."""
    n = values.shape[-1]
    v = torch.nn.functional.pad(values, (0, _up(n, 32) - n)).unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top).exponent - 1 - _EMAX[fmt], -127).clamp(min=-127)
    q = v * _power(-e)
    a = q.abs()
    if fmt == "mxfp4":
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    else:
        step = _power((torch.frexp(a).exponent - 1).clamp(min=-6) - 3)
    r = (torch.round(a / step) * step).clamp(max=_TOP[fmt])
    return torch.copysign(r, q), e


def _through_blocks(values, fmt):
    level, e = _to_blocks(values, fmt)
    return (level * _power(e)).flatten(-2)[..., :values.shape[-1]]


def _decode(codes, scales, n, fmt):
    if fmt == "mxfp4":
        level = _levels4()[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    else:
        level = codes.view(torch.float8_e4m3fn).float()
    nb = _up(n, 32) // 32
    return (level.unflatten(-1, (nb, 32)) * _power(scales[:, :nb].int() - 127)[..., None]).flatten(-2)[:, :n]


def _plain(s):
    op = s["op"]
    if op == "product":
        A = _decode(s["A"], s["As"], s["k"], s["a"])
        B = _decode(s["B"], s["Bs"], s["k"], s["b"])
        return {"C": (A @ B.t()).to(_TYPE[s["out"]])}
    if op == "objective":
        Y = s["Y"]
        err = Y - _through_blocks(Y, s["format"])
        c = 1.0 / s["tokens"] if s["reduce"] == "mean" else 1.0
        loss = err.double().square().sum((1, 2)) * (c / s["n"])
        return {"loss": loss.float(), "dY": (err * (2.0 * c / s["n"])).to(_TYPE[s["grad"]])}
    dtype = _TYPE[s["x"]]
    if op == "quantize":
        return {"values": _through_blocks(s["X"].float(), s["format"]).to(dtype)}
    h = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(dtype)
    w = h.double()                           # 64 bits: values next to the border between two codes
    y = w / torch.sqrt(w.square().mean(-1, keepdim=True) + _EPS)
    if s["g"] is not None:
        y = y * s["g"].double()
    out = {"values": _through_blocks(y.float(), s["format"]).to(dtype)}
    return out if s["R"] is None else {"H": h, **out}


# ---- the library's calls

_kept = {}


def _library():
    """A context with its status word's memory for each stream that passes run on: a context's calls go to the stream that was the current one
    when it was made.  (Raw handles, since torch.cuda.current_stream() takes 2.6 us, half of a call.)"""
    device = torch._C._cuda_getDevice()
    key = (device, torch._C._cuda_getCurrentRawStream(device))
    lib = _kept.get(key)
    if lib is None:
        from paper_2511_04063_amd import binding as B
        ctx = B.Context()
        ctx.ensure_workspace(1, 1, 1, B.DQ_F32)
        lib = _kept[key] = dict(B=B, ctx=ctx, type={"bf16": B.DQ_BF16, "f32": B.DQ_F32}, format={"mxfp4": B.DQ_MXFP4, "mxfp8": B.DQ_MXFP8},
                                objective={"mxfp4": B.DQ_OBJ_MXFP4, "mxfp8": B.DQ_OBJ_MXFP8},
                                reduce={"mean": B.DQ_REDUCE_TOKEN_MEAN, "sum": B.DQ_REDUCE_SUM})
    return lib


def _calls(s):
    lib = _library()
    ctx, op = lib["ctx"], s["op"]
    if op == "product":
        ctx.dq_gemm_mx(s["m"], s["n"], s["k"], lib["format"][s["a"]], s["A"], s["As"], lib["format"][s["b"]], s["B"], s["Bs"], s["C"],
                       lib["type"][s["out"]])
        return {"C": s["C"]}
    if op == "objective":
        ctx.dq_objective_loss_grad(lib["objective"][s["format"]], 4, s["Y"], lib["reduce"][s["reduce"]], s["loss"], s["dY"],
                                   lib["type"][s["grad"]])
        return {"loss": s["loss"], "dY": s["dY"]}
    t, f = lib["type"][s["x"]], lib["format"][s["format"]]
    if op == "quantize":
        ctx.dq_mx_quantize(s["X"], t, f, s["codes"], s["scales"])
    else:
        ctx.dq_mx_rms_norm(s["X"], t, s["R"], s["H"], s["g"], _EPS, f, s["codes"], s["scales"])
    ctx.dq_mx_dequantize(f, s["codes"], s["scales"], s["values"], t)
    return {"values": s["values"]} if s.get("H") is None else {"H": s["H"], "values": s["values"]}


def run(state):
    return _calls(state) if own else _plain(state)


def work(case):
    """Inputs read once and outputs written once."""
    op = case["op"]
    size = {"bf16": 2, "f32": 4}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        held = {"mxfp4": 17 / 32, "mxfp8": 33 / 32}
        return {"bytes": m * k * held[case["a"]] + n * k * held[case["b"]] + m * n * size[case["out"]], "flops": 2.0 * m * n * k}
    if op == "objective":
        count = case["b"] * case["tokens"] * case["n"]
        return {"bytes": count * (4 + size[case["grad"]]) + 4 * case["b"], "flops": 8.0 * count}
    count = case["tokens"] * case["n"]
    moved = 2 if op == "quantize" else 4 if case["residual"] else 2
    return {"bytes": count * moved * size[case["x"]] + (4 * case["n"] if case.get("gain") else 0), "flops": (6.0 if op == "quantize" else 12.0) * count}


# ---- the definition in 64 bits

def _grid(fmt):
    """Representable magnitudes in the order of their codes."""
    bits, bias = (1, 1) if fmt == "mxfp4" else (3, 7)
    count = 8 if fmt == "mxfp4" else 127
    values = []
    for code in range(count):
        e, f = code >> bits, code & ((1 << bits) - 1)
        values.append(math.ldexp(f, 1 - bias - bits) if e == 0 else math.ldexp((1 << bits) + f, e - bias - bits))
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def _nearest(values, fmt):
    """Every value of the blocks of the last axis in place of its nearest representable one, by looking it up between the midpoints."""
    n = values.shape[-1]
    out = torch.empty_like(values)
    powers = torch.tensor([2.0 ** i for i in range(-128, 128)], dtype=torch.float64, device="cuda")
    grid = _grid(fmt)
    mid = (grid[1:] + grid[:-1]) / 2
    for first in range(0, n, 32):
        v = values[..., first:first + 32]
        top = v.abs().amax(-1)
        e = (torch.bucketize(top, powers, right=True) - 1 - 128 - _EMAX[fmt]).clamp(min=-127)
        scale = powers[e + 128].unsqueeze(-1)
        a = v.abs() / scale
        below = torch.bucketize(a, mid)                      # midpoints below a: a tie stays with the lower code
        tie = mid[below.clamp(max=mid.numel() - 1)] == a
        code = torch.where(tie & (below % 2 == 1), below + 1, below)
        out[..., first:first + 32] = torch.sign(v) * grid[code.clamp(max=grid.numel() - 1)] * scale
    return out


def _meaning(codes, scales, n, fmt):
    """The values of a stored matrix."""
    grid = _grid(fmt)
    signed = torch.cat((grid, -grid)) if fmt == "mxfp4" else torch.cat((grid, torch.zeros(1, dtype=grid.dtype, device="cuda"), -grid))
    byte = codes.long()
    code = torch.stack((byte % 16, byte // 16), -1).reshape(codes.shape[0], -1) if fmt == "mxfp4" else byte
    powers = torch.tensor([2.0 ** (i - 127) for i in range(255)], dtype=torch.float64, device="cuda")
    per = powers[scales.long()].repeat_interleave(32, dim=1)[:, :code.shape[1]]
    return (signed[code] * per)[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        return {"C": torch.mm(_meaning(s["A"], s["As"], s["k"], s["a"]), _meaning(s["B"], s["Bs"], s["k"], s["b"]).t().contiguous())}
    if op == "objective":
        Y = s["Y"].double()
        err = Y - _nearest(Y, s["format"])
        per_token = (err ** 2).sum(-1) / s["n"]
        loss = per_token.mean(-1) if s["reduce"] == "mean" else per_token.sum(-1)
        return {"loss": loss, "dY": 2.0 * err / (s["n"] * (s["tokens"] if s["reduce"] == "mean" else 1))}
    X = s["X"].double()
    if op == "quantize":
        return {"values": _nearest(X, s["format"])}
    if s["R"] is not None:
        X = (X + s["R"].double()).to(_TYPE[s["x"]]).double()        # the norm is that of the sum as it is stored
    y = X * torch.rsqrt((X * X).sum(-1) / s["n"] + _EPS).unsqueeze(-1)
    if s["g"] is not None:
        y = y * s["g"].double()
    values = _nearest(y.float().double(), s["format"])              # quantised is the norm's result in fp32
    return {"values": values} if s["R"] is None else {"H": X, "values": values}
