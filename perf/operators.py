"""The operators around a block-circulant adapter in a fine-tuned layer, as cases that can be timed and compared.

Six kinds of case:

* ``act8``            a row of activations into its 8-bit checkpoint and back.
* ``norm_forward``    layer norm for inference.
* ``norm_train``      layer norm forward and backward: y, dx and the weight's and bias's gradients.  With ``residual``
                      the norm's input is the sum of two tensors; with ``checkpoint`` the backward has that input as an
                      8-bit checkpoint only.
* ``linear_forward``  y = act(x W^T + b) + r for inference.  ``pitch``: x is a slice of rows that are this much longer.
* ``linear_train``    the product forward and backward: y, dx (to which the gradient of another branch is added), and,
                      unless W is ``frozen``, dW and db.  The pre-activation is kept as an 8-bit checkpoint.
* ``linear_backward`` the backward alone, from a checkpoint in hand.

The 8-bit format: blocks of 32 consecutive values of a row share a power of two 2^e, the least with
max|x| <= 127 * 2^e, and each value is rint(x / 2^e) in int8.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ITEM = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32
EPS = 1e-5


def listed():
    return [
        # the checkpoint of a small layer's short batch: latency
        {"name": "act8_f32_128x256", "kind": "act8", "dtype": "f32", "tokens": 128, "n": 256},
        # a 4096-wide decoder's activations, 16384 tokens
        {"name": "act8_bf16_16384x4096", "kind": "act8", "dtype": "bf16", "tokens": 16384, "n": 4096},
        # serving: the norm of one token of a 4096-wide decoder
        {"name": "norm_forward_bf16_1x4096", "kind": "norm_forward", "dtype": "bf16", "tokens": 1, "n": 4096},
        # an odd width in float32, nothing kept but the input
        {"name": "norm_train_f32_2045x769", "kind": "norm_train", "dtype": "f32", "tokens": 2045, "n": 769,
         "residual": False, "checkpoint": False},
        # an encoder's add-and-norm, 4096 tokens of width 768
        {"name": "norm_train_bf16_4096x768", "kind": "norm_train", "dtype": "bf16", "tokens": 4096, "n": 768,
         "residual": True, "checkpoint": True},
        # the same in a 4096-wide layer over 16384 tokens
        {"name": "norm_train_bf16_16384x4096", "kind": "norm_train", "dtype": "bf16", "tokens": 16384, "n": 4096,
         "residual": True, "checkpoint": True},
        # serving: one token through a 4096-wide projection whose adapter's output is the residual
        {"name": "linear_forward_bf16_1_4096x4096", "kind": "linear_forward", "dtype": "bf16", "tokens": 1, "d_in": 4096,
         "d_out": 4096, "activation": "none", "residual": True, "pitch": 0},
        # a few dozen tokens, float16, 1024 -> 4096
        {"name": "linear_forward_f16_61_1024x4096", "kind": "linear_forward", "dtype": "f16", "tokens": 61, "d_in": 1024,
         "d_out": 4096, "activation": "gelu", "residual": False, "pitch": 64},
        # an encoder's 768-wide projection, trained whole
        {"name": "linear_train_bf16_4096_768x768", "kind": "linear_train", "dtype": "bf16", "tokens": 4096, "d_in": 768,
         "d_out": 768, "activation": "gelu", "frozen": False},
        # float32, ragged tokens, the backward of a 1024 -> 768 layer
        {"name": "linear_backward_f32_1021_1024x768", "kind": "linear_backward", "dtype": "f32", "tokens": 1021,
         "d_in": 1024, "d_out": 768, "activation": "silu", "frozen": False},
        # fine-tuning: a frozen 4096-wide projection, ragged tokens
        {"name": "linear_train_bf16_2045_4096x4096", "kind": "linear_train", "dtype": "bf16", "tokens": 2045,
         "d_in": 4096, "d_out": 4096, "activation": "silu", "frozen": True},
        # the largest: 4096 -> 8192 over 8192 tokens, every gradient
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
    """One more case of the same ranges: norms and checkpoints of 1 to 16384 rows of 32 to 8192 values (at most 2^26),
    products of 1 to 16384 tokens, 64 to 8192 wide, of at most 2^38 multiply-adds each."""
    kind = rng.choice(["act8", "norm_forward", "norm_train", "norm_train", "linear_forward", "linear_forward",
                       "linear_train", "linear_train", "linear_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("act8", "norm_forward", "norm_train"):
        n = _width(rng, 32, 8192)
        case = {"kind": kind, "dtype": dtype, "tokens": _log_int(rng, 1, min(16384, 2**26 // n)), "n": n}
        if kind == "norm_train":
            case["residual"] = rng.random() < 0.5
            case["checkpoint"] = rng.random() < 0.6
        return case
    d_in, d_out = _width(rng, 64, 8192), _width(rng, 64, 8192)
    # (float32 products take sixteen times as long on the matrix cores)
    most = (2**34 if dtype == "f32" else 2**38) // (d_in * d_out)
    case = {"kind": kind, "dtype": dtype, "tokens": _log_int(rng, 1, min(16384, max(1, most))), "d_in": d_in,
            "d_out": d_out, "activation": rng.choice(["none", "relu", "gelu", "silu"])}
    if kind == "linear_forward":
        case["residual"] = rng.random() < 0.5
        case["pitch"] = rng.choice([0, 0, 8, 64])
        return case
    if kind == "linear_train" and dtype == "f32":
        case["activation"] = "none"  # a float32 pre-activation is kept exactly or not at all
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


def prepare(case, seed):
    g = _generator(seed)
    kind, dt, T = case["kind"], DTYPES[case["dtype"]], case["tokens"]
    state = {"kind": kind}

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def checkpoint(n):
        return empty(T, n, dtype=torch.int8), empty(T, -(-n // BLOCK), dtype=torch.uint8)

    if kind in ("act8", "norm_forward", "norm_train"):
        n = case["n"]
        state["x"] = _hidden(g, T, n, dt)
        if kind == "act8":
            state.update(codes=checkpoint(n), out=empty(T, n))
            return state
        state.update(weight=1.0 + 0.1 * _normal(g, n), bias=0.1 * _normal(g, n), y=empty(T, n))
        if kind == "norm_train":
            state.update(mean=empty(T, dtype=torch.float32), rstd=empty(T, dtype=torch.float32),
                         residual=_hidden(g, T, n, dt) if case["residual"] else None,
                         codes=checkpoint(n) if case["checkpoint"] else None, dy=_normal(g, T, n).to(dt), dx=empty(T, n),
                         dweight=empty(n, dtype=torch.float32), dbias=empty(n, dtype=torch.float32))
        return state
    d_in, d_out = case["d_in"], case["d_out"]
    x = _normal(g, T, d_in + case.get("pitch", 0)).to(dt)
    # weights that keep the variance
    state.update(x=x[:, :d_in], w=(_normal(g, d_out, d_in) / math.sqrt(d_in)).to(dt), activation=case["activation"])
    if kind != "linear_backward":
        state.update(bias=(0.5 * _normal(g, d_out)).to(dt), y=empty(T, d_out), residual=None)
    if kind == "linear_forward":
        if case["residual"]:
            state["residual"] = _normal(g, T, d_out).to(dt)
        return state
    state.update(dy=_normal(g, T, d_out).to(dt), add=_normal(g, T, d_in).to(dt), dx=empty(T, d_in), codes=None,
                 dw=None if case["frozen"] else empty(d_out, d_in), db=None if case["frozen"] else empty(d_out))
    if case["activation"] != "none":
        state["codes"] = _encode(_normal(g, T, d_out)) if kind == "linear_backward" else checkpoint(d_out)
    return state


# ---------------------------------------------------------------------------------------------
# the operators in their plain form


def _power(byte):
    """2^(byte - 127) as float32 (NaN for 255)."""
    b = byte.to(torch.int32)
    bits = torch.where(b == 0, torch.full_like(b, 0x00400000), b << 23)
    return torch.where(b == 255, torch.full_like(bits, 0x7FC00000), bits).view(torch.float32)


def _encode(x):
    """The checkpoint of float32 rows: codes (int8) and scale bytes (uint8)."""
    rows, n = x.shape
    blocks = -(-n // BLOCK)
    b = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).reshape(rows, blocks, BLOCK)
    amax = b.abs().amax(dim=2)
    fine = torch.isfinite(amax)
    m, k = torch.frexp(torch.where(fine, amax, torch.ones_like(amax)))
    e = torch.where(m <= 127.0 / 128.0, k - 7, k - 6)
    e = torch.where(amax == 0, torch.full_like(e, -127), e).clamp(min=-127)
    codes = torch.round(torch.where(fine.unsqueeze(2), b, torch.zeros_like(b)) * _power(127 - e).unsqueeze(2))
    byte = torch.where(fine, e + 127, torch.full_like(e, 255))
    return codes.to(torch.int8).reshape(rows, blocks * BLOCK)[:, :n].contiguous(), byte.to(torch.uint8)


def _decode(codes, scales):
    """The float32 values that a checkpoint stands for."""
    return codes.float() * _power(scales).repeat_interleave(BLOCK, dim=1)[:, : codes.shape[1]]


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


def _plain_norm(s):
    dt = s["x"].dtype
    u = s["x"].float()
    if s.get("residual") is not None:
        u = u + s["residual"].float()
    mean = u.mean(dim=1, keepdim=True)
    centred = u - mean
    rstd = 1 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    y = (centred * rstd * s["weight"] + s["bias"]).to(dt)
    if s["kind"] == "norm_forward":
        return {"y": y}
    if s["codes"] is not None:
        centred = _decode(*_encode(u)) - mean
    xhat, dy = centred * rstd, s["dy"].float()
    g = dy * s["weight"]
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return {"y": y, "dx": dx.to(dt), "dweight": (dy * xhat).sum(dim=0), "dbias": dy.sum(dim=0)}


def _plain_linear(s):
    dt, name, out = s["x"].dtype, s["activation"], {}
    x, w = s["x"].float(), s["w"].float()
    codes = s.get("codes")
    if s["kind"] != "linear_backward":
        z = x @ w.t() + s["bias"].float()
        y = _act(name, z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out["y"] = y.to(dt)
        if s["kind"] == "linear_forward":
            return out
        if codes is not None:
            codes = _encode(z)
    dz = s["dy"].float()
    if codes is not None:
        dz = dz * _act_slope(name, _decode(*codes))
    out["dx"] = (dz @ w + s["add"].float()).to(dt)
    if s["dw"] is not None:
        out["dw"] = (dz.t() @ x).to(dt)
        out["db"] = dz.sum(dim=0).to(dt)
    return out


# ---------------------------------------------------------------------------------------------
# the framework's operators


def _own(s):
    from paper_2511_01385_amd import api

    kind = s["kind"]
    if kind == "act8":
        api.act8_quantize(s["x"], *s["codes"])
        return {"values": api.act8_dequantize(*s["codes"], s["out"])}
    if kind == "norm_forward":
        return {"y": api.layer_norm_forward(s["x"], s["weight"], s["bias"], s["y"], eps=EPS)}
    if kind == "norm_train":
        api.layer_norm_forward(s["x"], s["weight"], s["bias"], s["y"], residual=s["residual"], mean=s["mean"],
                               rstd=s["rstd"], checkpoint=s["codes"], eps=EPS)
        if s["codes"] is not None:
            api.layer_norm_backward(s["dy"], s["codes"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"],
                                    s["dbias"])
        else:
            api.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"],
                                    s["dbias"], residual=s["residual"])
        return {k: s[k] for k in ("y", "dx", "dweight", "dbias")}
    out = {}
    if kind != "linear_backward":
        out["y"] = api.linear_forward(s["x"], s["w"], s["y"], bias=s["bias"], activation=s["activation"],
                                      residual=s["residual"], checkpoint=s.get("codes"))
        if kind == "linear_forward":
            return out
    api.linear_backward(s["dy"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], db=s["db"], activation=s["activation"],
                        checkpoint=s["codes"], add=s["add"])
    out["dx"] = s["dx"]
    if s["dw"] is not None:
        out.update(dw=s["dw"], db=s["db"])
    return out


def run(state):
    if own:
        return _own(state)
    kind = state["kind"]
    if kind == "act8":
        return {"values": _decode(*_encode(state["x"].float())).to(state["x"].dtype)}
    return _plain_norm(state) if kind in ("norm_forward", "norm_train") else _plain_linear(state)


def work(case):
    s, T, kind = ITEM[case["dtype"]], case["tokens"], case["kind"]
    held = 1 + 1 / BLOCK  # bytes of a checkpoint's value
    if kind == "act8":
        return {"bytes": T * case["n"] * (2 * s + 2 * held), "flops": 4 * T * case["n"]}
    if kind in ("norm_forward", "norm_train"):
        n = case["n"]
        if kind == "norm_forward":
            return {"bytes": 2 * T * n * s + 8 * n, "flops": 8 * T * n}
        inputs = 2 if case["residual"] else 1
        kept = 2 * held if case["checkpoint"] else inputs * s  # written and read, or the inputs read again
        return {"bytes": T * (n * ((inputs + 3) * s + kept) + 16) + 20 * n, "flops": 24 * T * n}
    d_in, d_out = case["d_in"], case["d_out"]
    product, x, z, w = 2.0 * T * d_in * d_out, T * d_in * s, T * d_out * s, d_in * d_out * s
    kept = 0 if case["activation"] == "none" else T * d_out * held
    forward = {"bytes": x + z + w + d_out * s, "flops": product}
    if kind == "linear_forward":
        forward["bytes"] += z if case["residual"] else 0
        return forward
    backward = {"bytes": z + kept + w + 2 * x, "flops": product}
    if not case["frozen"]:
        backward["bytes"] += x + w + d_out * s
        backward["flops"] += product
    if kind == "linear_backward":
        return backward
    return {"bytes": forward["bytes"] + kept + backward["bytes"], "flops": forward["flops"] + backward["flops"]}


# ---------------------------------------------------------------------------------------------
# the same results in 64 bits from the definitions


def _two_to(k):
    """2^k as float64, to the bit (a power function is not)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_checkpoint(u):
    """Every value of float64 rows replaced by what its 8-bit checkpoint stands for."""
    out = torch.empty_like(u)
    whole = u.shape[1] // BLOCK * BLOCK
    for part, width in ((slice(0, whole), BLOCK), (slice(whole, None), u.shape[1] - whole)):
        v = u[:, part]
        if v.numel() == 0:
            continue
        v = v.reshape(u.shape[0], -1, width)
        top = v.abs().max(dim=2, keepdim=True).values
        unit = torch.frexp(top / torch.full_like(top, 127))  # (a division by a number is a product with its inverse)
        # 2^exponent >= top / 127, or half of it where top / 127 is a power of two itself
        power = torch.where(unit.mantissa == 0.5, unit.exponent - 1, unit.exponent).clamp(min=-127)
        step = _two_to(power)
        out[:, part] = (torch.round(v / step) * step).reshape(u.shape[0], -1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "act8":
        return {"values": _exact_checkpoint(s["x"].double())}
    if kind in ("norm_forward", "norm_train"):
        w, b = s["weight"].double(), s["bias"].double()
        u = s["x"].double()
        if s.get("residual") is not None:
            u = u + s["residual"].double()
        mean = u.mean(1, True)
        sigma = torch.sqrt(u.var(1, unbiased=False, keepdim=True) + EPS)
        y = w * (u - mean) / sigma + b
        if kind == "norm_forward":
            return {"y": y}
        if s["codes"] is not None:
            # the checkpoint is of the 32-bit sum
            u = _exact_checkpoint(u.float().double())
        xhat, dy = (u - mean) / sigma, s["dy"].double()
        g = dy * w
        dx = (g - g.mean(1, True) - xhat * (g * xhat).mean(1, True)) / sigma
        return {"y": y, "dx": dx, "dweight": torch.linalg.vecdot(dy, xhat, dim=0), "dbias": dy.sum(0)}
    x, w, name, out = s["x"].double(), s["w"].double(), s["activation"], {}
    if kind == "linear_backward":
        z = None
        if s["codes"] is not None:
            codes, scales = s["codes"]
            power = _two_to(scales.int() - 127)
            z = codes.double() * power[:, torch.arange(codes.shape[1], device=codes.device) // BLOCK]
    else:
        z = torch.addmm(s["bias"].double(), x, w.t())
        soft = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
                "silu": torch.nn.functional.silu}[name]
        out["y"] = soft(z) if s["residual"] is None else soft(z) + s["residual"].double()
        if kind == "linear_forward":
            return out
        z = _exact_checkpoint(z)
    dz = s["dy"].double()
    if name == "relu":
        dz = torch.where(z > 0, dz, torch.zeros_like(dz))
    elif name == "gelu":
        dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    elif name == "silu":
        dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
    out["dx"] = torch.addmm(s["add"].double(), dz, w)
    if s["dw"] is not None:
        out.update(dw=torch.mm(dz.t().contiguous(), x), db=dz.sum(0))
    return out
