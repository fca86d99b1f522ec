"""RMS norm and the dense product in 8-bit floating point, as cases that can be timed and compared.

Seven kinds of case:

* ``quantize``        a matrix into 8 bits and back: its rows, its columns (the rows of its transpose), or both.
* ``norm_forward``    RMS norm for inference: the sum with the residual, and the normalised rows.
* ``norm_train``      RMS norm forward and backward: the sum, y, dx (to which the residual stream's gradient is added) and
                      the weight's gradient.  With ``checkpoint`` the backward has the sum as an 8-bit checkpoint only.
* ``norm_linear``     serving: the norm's output in 8 bits and the product that takes it.
* ``linear_forward``  y = act(x W^T + b) + r of operands in 8 bits.
* ``linear_train``    a training pass: x (and W, unless it is ``frozen``) quantized, the product forward and backward:
                      y, dx (to which the gradient of another branch is added), dW and db unless W is frozen.
                      The pre-activation is kept as an int8 checkpoint.
* ``linear_backward`` the backward alone, of dy and of what a forward has left.

The 8-bit floating point format: blocks of 128 consecutive values of a row (the last may be short), or tiles of 128 x 128
of a weight, share a power of two 2^e, the least with max|x| <= 448 * 2^e; each value is x / 2^e rounded to e4m3.
A row of codes starts at a multiple of 16 bytes, one of scales at a multiple of 4.  The int8 checkpoint: blocks of 32, rint(x / 2^e), max|x| <= 127 * 2^e.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ITEM = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
CK_BLOCK = 32
EPS = 1e-6


def listed():
    return [
        # the 8-bit form of a small layer's weight, both ways, in tiles
        {"name": "quantize_f32_256x384", "kind": "quantize", "dtype": "f32", "rows": 256, "n": 384, "tiles": True,
         "columns": True},
        # activations of 8192 tokens, 4096 wide, for the forward (rows) and the weight's gradient (columns)
        {"name": "quantize_bf16_8192x4096", "kind": "quantize", "dtype": "bf16", "rows": 8192, "n": 4096, "tiles": False,
         "columns": True},
        # serving: one token of a 4096-wide decoder
        {"name": "norm_forward_bf16_1x4096", "kind": "norm_forward", "dtype": "bf16", "tokens": 1, "n": 4096},
        # an odd width in float32
        {"name": "norm_train_f32_2045x769", "kind": "norm_train", "dtype": "f32", "tokens": 2045, "n": 769,
         "checkpoint": False},
        # a 4096-wide decoder layer over 16384 tokens, the norm's input kept in 8 bits
        {"name": "norm_train_bf16_16384x4096", "kind": "norm_train", "dtype": "bf16", "tokens": 16384, "n": 4096,
         "checkpoint": True},
        # serving: one token through norm and projection of a 4096-wide decoder
        {"name": "norm_linear_bf16_1_4096x4096", "kind": "norm_linear", "dtype": "bf16", "tokens": 1, "d_in": 4096,
         "d_out": 4096},
        # a prompt's tokens through the same, ragged
        {"name": "norm_linear_bf16_1021_4096x4096", "kind": "norm_linear", "dtype": "bf16", "tokens": 1021, "d_in": 4096,
         "d_out": 4096},
        # a few dozen tokens, float16, 1024 -> 4096
        {"name": "linear_forward_f16_61_1024x4096", "kind": "linear_forward", "dtype": "f16", "tokens": 61, "d_in": 1024,
         "d_out": 4096, "activation": "gelu", "residual": False},
        # an odd layer with a float32 result
        {"name": "linear_forward_f32_1021_1001x771", "kind": "linear_forward", "dtype": "f32", "tokens": 1021, "d_in": 1001,
         "d_out": 771, "activation": "none", "residual": True},
        # the backward of an encoder's 768-wide projection, ragged tokens, every gradient
        {"name": "linear_backward_bf16_4093_768x768", "kind": "linear_backward", "dtype": "bf16", "tokens": 4093,
         "d_in": 768, "d_out": 768, "activation": "gelu", "frozen": False},
        # fine-tuning: a frozen 4096-wide projection, ragged tokens
        {"name": "linear_train_bf16_2045_4096x4096", "kind": "linear_train", "dtype": "bf16", "tokens": 2045,
         "d_in": 4096, "d_out": 4096, "activation": "silu", "frozen": True},
        # the largest: 4096 -> 8192 over 8192 tokens, every gradient, W quantized anew
        {"name": "linear_train_bf16_8192_4096x8192", "kind": "linear_train", "dtype": "bf16", "tokens": 8192,
         "d_in": 4096, "d_out": 8192, "activation": "gelu", "frozen": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A feature width: most are multiples of 64, some of 8, a few odd."""
    n = _log_int(rng, lo, hi)
    how = rng.random()
    return max(lo, n // 64 * 64 if how < 0.6 else n // 8 * 8 if how < 0.85 else n)


def draw(rng):
    """One more case of the same ranges: norms and matrices of 1 to 16384 rows of 32 to 8192 values (at most 2^26),
    products of 1 to 16384 tokens, 64 to 8192 wide, of at most 2^38 multiply-adds each."""
    kind = rng.choice(["quantize", "norm_forward", "norm_train", "norm_linear", "linear_forward", "linear_forward",
                       "linear_train", "linear_train", "linear_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("quantize", "norm_forward", "norm_train"):
        n = _width(rng, 32, 8192)
        rows = _log_int(rng, 1, min(16384, 2**26 // n))
        if kind == "quantize":
            return {"kind": kind, "dtype": dtype, "rows": rows, "n": n, "tiles": rng.random() < 0.4,
                    "columns": rng.random() < 0.6}
        case = {"kind": kind, "dtype": dtype, "tokens": rows, "n": n}
        if kind == "norm_train":
            case["checkpoint"] = rng.random() < 0.5
        return case
    d_in, d_out = _width(rng, 64, 8192), _width(rng, 64, 8192)
    case = {"kind": kind, "dtype": dtype, "tokens": _log_int(rng, 1, min(16384, max(1, 2**38 // (d_in * d_out)))),
            "d_in": d_in, "d_out": d_out}
    if kind == "norm_linear":
        # (a last bit of a float32 norm can move a value to the next 8-bit number, which a float32 product would show)
        case["dtype"] = "f16" if dtype == "f32" else dtype
        return case
    # (what a float32 gradient is made of is the same on every path only where no activation's bits come in)
    case["activation"] = "none" if dtype == "f32" else rng.choice(["none", "relu", "gelu", "silu"])
    if kind == "linear_forward":
        case["residual"] = rng.random() < 0.5
    else:
        case["frozen"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------------------------
# inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _hidden(g, tokens, n, dt):
    """A hidden state: unit variance, features with their own mean, and a few of ten times the size, as trained models have."""
    size = torch.where(torch.rand(n, generator=g, device="cuda") < 0.01, 10.0, 1.0)
    return ((_normal(g, tokens, n) + 0.3 * _normal(g, n)) * size).to(dt)


def _weight(g, d_out, d_in):
    """Weights that keep the variance."""
    return _normal(g, d_out, d_in) / math.sqrt(d_in)


def _empty8(rows, n, tiles=False):
    """Room for rows x n values in 8 bits."""
    codes = torch.empty(rows, -(-n // 16) * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :n]
    blocks, bands = -(-n // BLOCK), -(-rows // BLOCK) if tiles else rows
    return codes, torch.empty(bands, -(-blocks // 4) * 4, dtype=torch.uint8, device="cuda")[:, :blocks]


def _filled8(x, tiles=False):
    held = _empty8(*x.shape, tiles)
    for to, v in zip(held, _encode8(x, tiles)):
        to.copy_(v)
    return held


def prepare(case, seed):
    g = _generator(seed)
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    state = {"kind": kind}

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def checkpoint(rows, n):
        return empty(rows, n, dtype=torch.int8), empty(rows, -(-n // CK_BLOCK), dtype=torch.uint8)

    if kind == "quantize":
        rows, n, tiles = case["rows"], case["n"], case["tiles"]
        state.update(x=_weight(g, rows, n).to(dt) if tiles else _hidden(g, rows, n, dt), tiles=tiles,
                     rows=_empty8(rows, n, tiles), columns=_empty8(n, rows, tiles) if case["columns"] else None,
                     out=empty(rows, n), out_columns=empty(n, rows))
        return state
    T = case["tokens"]
    if kind in ("norm_forward", "norm_train", "norm_linear"):
        n = case["d_in"] if kind == "norm_linear" else case["n"]
        state.update(x=_normal(g, T, n).to(dt), residual=_hidden(g, T, n, dt), weight=1.0 + 0.1 * _normal(g, n),
                     summed=empty(T, n))
        if kind == "norm_linear":
            state.update(x8=_empty8(T, n), w=_filled8(_weight(g, case["d_out"], n), True), y=empty(T, case["d_out"]))
            return state
        state["y"] = empty(T, n)
        if kind == "norm_train":
            state.update(rstd=empty(T, dtype=torch.float32), codes=checkpoint(T, n) if case["checkpoint"] else None,
                         dy=_normal(g, T, n).to(dt), add=_normal(g, T, n).to(dt), dx=empty(T, n),
                         dweight=empty(n, dtype=torch.float32))
        return state
    d_in, d_out = case["d_in"], case["d_out"]
    x, w = _hidden(g, T, d_in, dt), _weight(g, d_out, d_in).to(dt)
    state.update(activation=case["activation"], codes=None, residual=None)
    if kind != "linear_backward":
        state.update(bias=(0.5 * _normal(g, d_out)).to(dt), y=empty(T, d_out))
    if kind == "linear_forward":
        state.update(x8=_filled8(x.float()), w8=_filled8(w.float(), True))
        if case["residual"]:
            state["residual"] = _normal(g, T, d_out).to(dt)
        return state
    frozen = case["frozen"]
    state.update(frozen=frozen, dy=_normal(g, T, d_out).to(dt), add=_normal(g, T, d_in).to(dt), dx=empty(T, d_in),
                 dw=None if frozen else empty(d_out, d_in), db=None if frozen else empty(d_out))
    if kind == "linear_backward":
        state.update(w8t=_filled8(w.float().t(), True), x8t=None if frozen else _filled8(x.float().t()))
        if case["activation"] != "none":
            state["codes"] = _encode(_normal(g, T, d_out))
        return state
    state.update(x=x, x8=_empty8(T, d_in), x8t=None if frozen else _empty8(d_in, T))
    if frozen:
        state.update(w8=_filled8(w.float(), True), w8t=_filled8(w.float().t(), True))
    else:
        state.update(w=w, w8=_empty8(d_out, d_in, True), w8t=_empty8(d_in, d_out, True))
    if case["activation"] != "none":
        state["codes"] = checkpoint(T, d_out)
    return state


# ---------------------------------------------------------------------------------------------
# the operators in their plain form


def _power(byte):
    """2^(byte - 127) as float32 (NaN for 255)."""
    b = byte.to(torch.int32)
    bits = torch.where(b == 0, torch.full_like(b, 0x00400000), b << 23)
    return torch.where(b == 255, torch.full_like(bits, 0x7FC00000), bits).view(torch.float32)


def _exponent(amax, top):
    """The least e >= -127 with amax <= top * 2^e, for top = 127 (of int8) or 448 (of e4m3)."""
    m, k = torch.frexp(amax)
    e = torch.where(m <= 127.0 / 128.0, k - 7, k - 6) if top == 127 else torch.where(m <= 0.875, k - 9, k - 8)
    return torch.where(amax == 0, torch.full_like(e, -127), e).clamp(min=-127)


def _encode(x):
    """The int8 checkpoint of float32 rows: codes and scale bytes."""
    rows, n = x.shape
    blocks = -(-n // CK_BLOCK)
    b = torch.nn.functional.pad(x, (0, blocks * CK_BLOCK - n)).reshape(rows, blocks, CK_BLOCK)
    e = _exponent(b.abs().amax(dim=2), 127)
    codes = torch.round(b * _power(127 - e).unsqueeze(2))
    return codes.to(torch.int8).reshape(rows, blocks * CK_BLOCK)[:, :n].contiguous(), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    return codes.float() * _power(scales).repeat_interleave(CK_BLOCK, dim=1)[:, : codes.shape[1]]


def _encode8(x, tiles=False):
    """float32 rows in 8-bit floating point: codes and scale bytes, one for 128 values of a row or for a tile of 128 x 128."""
    rows, n = x.shape
    blocks, high = -(-n // BLOCK), BLOCK if tiles else 1
    bands = -(-rows // high)
    b = torch.nn.functional.pad(x, (0, blocks * BLOCK - n, 0, bands * high - rows)).reshape(bands, high, blocks, BLOCK)
    e = _exponent(b.abs().amax(dim=(1, 3)), 448)
    codes = (b * _power(127 - e)[:, None, :, None]).to(torch.float8_e4m3fn)
    return codes.reshape(bands * high, blocks * BLOCK)[:rows, :n], (e + 127).to(torch.uint8)


def _decode8(codes, scales):
    """The float32 values that they stand for."""
    power = _power(scales)
    if scales.shape[0] != codes.shape[0]:
        power = power.repeat_interleave(BLOCK, dim=0)[: codes.shape[0]]
    return codes.float() * power.repeat_interleave(BLOCK, dim=1)[:, : codes.shape[1]]


def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_quantize(s):
    x, dt = s["x"].float(), s["x"].dtype
    out = {"values": _decode8(*_encode8(x, s["tiles"])).to(dt)}
    if s["columns"] is not None:
        out["columns"] = _decode8(*_encode8(x.t(), s["tiles"])).to(dt)
    return out


def _plain_norm(s):
    dt = s["x"].dtype
    u = (s["x"].float() + s["residual"].float()).to(dt)
    out = {"summed": u}
    u = u.float()
    rstd = 1 / torch.sqrt((u * u).mean(dim=1, keepdim=True) + EPS)
    y = u * rstd * s["weight"]
    if s["kind"] == "norm_linear":
        out["y"] = (_decode8(*_encode8(y)) @ _decode8(*s["w"]).t()).to(dt)
        return out
    out["y"] = y.to(dt)
    if s["kind"] == "norm_forward":
        return out
    if s["codes"] is not None:
        u = _decode(*_encode(u))
    xhat, dy = u * rstd, s["dy"].float()
    g = dy * s["weight"]
    dx = rstd * (g - xhat * (g * xhat).mean(dim=1, keepdim=True)) + s["add"].float()
    out.update(dx=dx.to(dt), dweight=(dy * xhat).sum(dim=0))
    return out


def _plain_linear(s):
    name, codes, out = s["activation"], s["codes"], {}
    kind = s["kind"]
    dt = (s["dy"] if kind == "linear_backward" else s["y"]).dtype
    if kind == "linear_backward":
        w = _decode8(*s["w8t"]).t()
        xt = None if s["frozen"] else _decode8(*s["x8t"])
    else:
        if kind == "linear_forward":
            x, w = _decode8(*s["x8"]), _decode8(*s["w8"])
        else:
            x = _decode8(*_encode8(s["x"].float()))
            xt = None if s["frozen"] else _decode8(*_encode8(s["x"].float().t()))
            w = _decode8(*(s["w8"] if s["frozen"] else _encode8(s["w"].float(), True)))
        z = x @ w.t() + s["bias"].float()
        y = _act(name, z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out["y"] = y.to(dt)
        if kind == "linear_forward":
            return out
        if codes is not None:
            codes = _encode(z)
    dz = s["dy"].float()
    if codes is not None:
        dz = dz * _act_slope(name, _decode(*codes))
    out["dx"] = (_decode8(*_encode8(dz)) @ w + s["add"].float()).to(dt)
    if not s["frozen"]:
        out["dw"] = (_decode8(*_encode8(dz.t())) @ xt.t()).to(dt)
        out["db"] = dz.sum(dim=0).to(dt)
    return out


# ---------------------------------------------------------------------------------------------
# the framework's operators


def _own(s):
    from paper_2511_01385_amd import api

    kind = s["kind"]
    if kind == "quantize":
        api.fp8_quantize(s["x"], s["rows"], columns=s["columns"])
        out = {"values": api.fp8_dequantize(s["rows"], s["out"])}
        if s["columns"] is not None:
            out["columns"] = api.fp8_dequantize(s["columns"], s["out_columns"])
        return out
    if kind == "norm_linear":
        api.rms_norm_forward(s["x"], s["weight"], residual=s["residual"], summed=s["summed"], y8=s["x8"], eps=EPS)
        return {"summed": s["summed"], "y": api.linear_fp8_forward(s["x8"], s["w"], s["y"])}
    if kind in ("norm_forward", "norm_train"):
        if kind == "norm_forward":
            api.rms_norm_forward(s["x"], s["weight"], s["y"], residual=s["residual"], summed=s["summed"], eps=EPS)
            return {"summed": s["summed"], "y": s["y"]}
        api.rms_norm_forward(s["x"], s["weight"], s["y"], residual=s["residual"], summed=s["summed"], rstd=s["rstd"],
                             checkpoint=s["codes"], eps=EPS)
        api.rms_norm_backward(s["dy"], s["summed"] if s["codes"] is None else s["codes"], s["weight"], s["rstd"], s["dx"],
                              s["dweight"], add=s["add"])
        return {k: s[k] for k in ("summed", "y", "dx", "dweight")}
    out = {}
    if kind == "linear_train":
        api.fp8_quantize(s["x"], s["x8"], columns=s["x8t"])
        if not s["frozen"]:
            api.fp8_quantize(s["w"], s["w8"], columns=s["w8t"])
    if kind != "linear_backward":
        out["y"] = api.linear_fp8_forward(s["x8"], s["w8"], s["y"], bias=s["bias"], activation=s["activation"],
                                          residual=s["residual"], checkpoint=s["codes"])
        if kind == "linear_forward":
            return out
    api.linear_fp8_backward(s["dy"], s["x8t"], s["w8t"], dx=s["dx"], dw=s["dw"], db=s["db"], activation=s["activation"],
                            checkpoint=s["codes"], add=s["add"])
    out["dx"] = s["dx"]
    if not s["frozen"]:
        out.update(dw=s["dw"], db=s["db"])
    return out


def run(state):
    if own:
        return _own(state)
    kind = state["kind"]
    if kind == "quantize":
        return _plain_quantize(state)
    return _plain_norm(state) if kind.startswith("norm") else _plain_linear(state)


def work(case):
    s, kind = ITEM[case["dtype"]], case["kind"]
    held, kept = 1 + 1 / BLOCK, 1 + 1 / CK_BLOCK  # bytes of a value in 8-bit floating point, and in a checkpoint
    if kind == "quantize":
        each = case["rows"] * case["n"]
        ways = 2 if case["columns"] else 1
        return {"bytes": each * (s + ways * (2 * (1 if case["tiles"] else held) + s)), "flops": 4 * each * ways}
    T = case["tokens"]
    if kind in ("norm_forward", "norm_train"):
        n = case["n"]
        if kind == "norm_forward":
            return {"bytes": 4 * T * n * s + 4 * n, "flops": 5 * T * n}
        # the sum written and read, or a checkpoint in its stead
        reads = kept * 2 if case["checkpoint"] else s
        return {"bytes": T * (n * (7 * s + reads) + 8) + 12 * n, "flops": 18 * T * n}
    d_in, d_out = case["d_in"], case["d_out"]
    product, x, z, w = 2.0 * T * d_in * d_out, T * d_in, T * d_out, d_in * d_out
    if kind == "norm_linear":
        return {"bytes": 3 * x * s + 4 * d_in + w + z * s, "flops": product}
    forward = {"bytes": x * held + w + z * s + d_out * s, "flops": product}
    if kind == "linear_forward":
        forward["bytes"] += z * s if case["residual"] else 0
        return forward
    ck = 0 if case["activation"] == "none" else z * kept
    backward = {"bytes": z * s + ck + w + 2 * x * s, "flops": product}
    if not case["frozen"]:
        backward["bytes"] += x * held + w * s + d_out * s
        backward["flops"] += product
    if kind == "linear_backward":
        return backward
    # x as it comes, for the forward; W as it comes where it is trained; what the backward needs is written once
    forward["bytes"] += x * (s - held) + ck
    if not case["frozen"]:
        forward["bytes"] += w * (s - 1) + x * held + w
    return {"bytes": forward["bytes"] + backward["bytes"], "flops": forward["flops"] + backward["flops"]}


# ---------------------------------------------------------------------------------------------
# the same results in 64 bits from the definitions


def _two_to(k):
    """2^k as float64, to the bit (a power function is not)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_held(u, top, width, high=1):
    """Every value of float64 rows replaced by what it is held as: blocks of high x width, whose largest code is `top`."""
    out = torch.empty_like(u)
    rows, n = u.shape
    whole_r, whole_n = rows // high * high, n // width * width
    for r, h in ((slice(0, whole_r), high), (slice(whole_r, rows), rows - whole_r)):
        for c, w in ((slice(0, whole_n), width), (slice(whole_n, n), n - whole_n)):
            v = u[r, c]
            if v.numel() == 0:
                continue
            v = v.reshape(-1, h, v.shape[1] // w, w)
            most = v.abs().amax(dim=(1, 3), keepdim=True)
            unit = torch.frexp(most / torch.full_like(most, top))  # (a division by a number is a product with its inverse)
            # 2^exponent >= most / top, or half of it where most / top is a power of two itself
            step = _two_to(torch.where(unit.mantissa == 0.5, unit.exponent - 1, unit.exponent).clamp(min=-127))
            q = v / step
            if top == 127:
                q = torch.round(q)
            else:
                # e4m3: 8 steps from a power of two to the next, from 2^-6 on; below, multiples of 2^-9
                grain = _two_to((torch.frexp(q).exponent - 1).clamp(min=-6) - 3)
                q = torch.round(q / grain) * grain
            out[r, c] = (q * step).reshape(out[r, c].shape)
    return out


def _exact8(u, tiles=False):
    return _exact_held(u, 448, BLOCK, BLOCK if tiles else 1)


def _stands_for(held):
    """The float64 values of codes and scale bytes in hand."""
    codes, scales = held
    at = torch.arange(codes.shape[0], device=codes.device)
    band = at // BLOCK if scales.shape[0] != codes.shape[0] else at
    return codes.double() * _two_to(scales.int() - 127)[band][:, torch.arange(codes.shape[1], device=codes.device) // BLOCK]


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "quantize":
        x = s["x"].double()
        out = {"values": _exact8(x, s["tiles"])}
        if s["columns"] is not None:
            out["columns"] = _exact8(x.t().contiguous(), s["tiles"])
        return out
    if kind.startswith("norm"):
        w = s["weight"].double()
        # the sum is kept in the storage type: the norm is of that
        out = {"summed": (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()}
        u = out["summed"]
        sigma = torch.sqrt(torch.linalg.vecdot(u, u, dim=1).unsqueeze(1) / u.shape[1] + EPS)
        y = w * u / sigma
        if kind == "norm_linear":
            out["y"] = torch.mm(_exact8(y), _stands_for(s["w"]).t().contiguous())
            return out
        out["y"] = y
        if kind == "norm_forward":
            return out
        if s["codes"] is not None:
            u = _exact_held(u, 127, CK_BLOCK)
        xhat, dy = u / sigma, s["dy"].double()
        g = dy * w
        dx = (g - xhat * (g * xhat).mean(1, True)) / sigma + s["add"].double()
        out.update(dx=dx, dweight=torch.linalg.vecdot(dy, xhat, dim=0))
        return out
    name, out = s["activation"], {}
    z = None
    if kind == "linear_backward":
        w = _stands_for(s["w8t"]).t()
        xt = None if s["frozen"] else _stands_for(s["x8t"])
        if s["codes"] is not None:
            codes, scales = s["codes"]
            z = codes.double() * _two_to(scales.int() - 127)[:, torch.arange(codes.shape[1], device=codes.device) // CK_BLOCK]
    else:
        if kind == "linear_forward":
            x, w = _stands_for(s["x8"]), _stands_for(s["w8"])
        else:
            x = _exact8(s["x"].double())
            xt = None if s["frozen"] else _exact8(s["x"].double().t().contiguous())
            w = _stands_for(s["w8"]) if s["frozen"] else _exact8(s["w"].double(), True)
        z = torch.addmm(s["bias"].double(), x, w.t())
        soft = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
                "silu": torch.nn.functional.silu}[name]
        out["y"] = soft(z) if s["residual"] is None else soft(z) + s["residual"].double()
        if kind == "linear_forward":
            return out
        z = _exact_held(z, 127, CK_BLOCK)
    dz = s["dy"].double()
    if name == "relu":
        dz = torch.where(z > 0, dz, torch.zeros_like(dz))
    elif name == "gelu":
        dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    elif name == "silu":
        dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
    out["dx"] = torch.addmm(s["add"].double(), _exact8(dz), w)
    if not s["frozen"]:
        out.update(dw=torch.mm(_exact8(dz.t().contiguous()), xt.t()), db=dz.sum(0))
    return out
