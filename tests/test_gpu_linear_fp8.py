"""The product of operands in 8-bit floating point and its gradients against float64 (the bounds of _fp8.product_error)."""

import math

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import TYPES, UNIT, decode, encode, f64, matmul64, product_error, random_operand, value

pytestmark = pytest.mark.gpu


def normal(rows, n, seed, dtype, wider=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, n + wider, generator=g, device="cuda").to(TYPES[dtype])[:, :n]


def forward(tokens, d_in, d_out, dtype, tiles=True, pad=0, seed=0, spread=3):
    x, w = random_operand(tokens, d_in, seed, pad=pad, spread=spread), random_operand(d_out, d_in, seed + 1, tiles, pad, spread)
    y = torch.full((tokens, d_out + 3 * pad), 5.0, dtype=TYPES[dtype], device="cuda")
    api.linear_fp8_forward(x, w, y[:, :d_out])
    product_error(f64(y[:, :d_out]), value(x), value(w), dtype, what=f"{dtype} {tokens} {d_in}->{d_out}")
    assert (y[:, d_out:] == 5).all()
    return y


# few tokens; every cut of a stage and of a chunk; more than sixteen stages to a wave
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(1, 1, 1), (1, 16, 8), (2, 7, 5), (1, 4096, 256), (3, 127, 33), (16, 128, 64),
                                               (17, 129, 65), (32, 1000, 130), (33, 1001, 70), (64, 2100, 96), (5, 17000, 48),
                                               (64, 17025, 40), (1, 300, 8200), (40, 260, 8200)])
def test_few_tokens(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, tiles=tokens % 2 == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(65, 1, 3), (65, 15, 64), (100, 128, 33), (129, 130, 257), (300, 512, 300),
                                               (130, 1001, 771), (200, 4099, 130), (1021, 640, 512), (2000, 2048, 1000),
                                               (128, 9000, 128), (70, 33000, 40)])
def test_tiles(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, tiles=tokens % 2 == 0, pad=tokens % 3)


@pytest.mark.parametrize("tokens,d_in,d_out", [(4096, 384, 4096), (4096 + 77, 1000, 4096 + 130), (2500, 700, 8192), (8192, 129, 2048)])
def test_largest_tiles(tokens, d_in, d_out):
    forward(tokens, d_in, d_out, "bf16", pad=1)


# sizes that every tile, with its k whole or split, is the cheapest for in one type or another; rows, columns, chunks and stages
# that are cut, enough stages for the loop's steady part, and some without a cut
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(2045, 1001, 5000), (600, 2049, 5000), (600, 2048, 5000), (2560, 1001, 2050),
                                               (2560, 1024, 2048), (2045, 1291, 4100), (4096, 2048, 4096), (3000, 1001, 129),
                                               (3000, 3001, 129), (1300, 1001, 777), (1300, 2049, 777), (1300, 1291, 777),
                                               (257, 6000, 129), (130, 6000, 129), (600, 1001, 5000), (130, 6000, 4100),
                                               (1000, 4097, 520)])
def test_every_tile(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, tiles=d_in % 2 == 0, pad=d_in % 3, spread=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(700, 3000, 770), (100, 3000, 1000), (300, 3000, 770), (100, 100, 129),
                                               (100, 100, 3000), (45, 1030, 700)])
def test_gradients_in_one_launch_and_two(dtype, tokens, d_in, d_out):
    backward(tokens, d_in, d_out, dtype, add=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 40, 65, 200])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_epilogue(dtype, tokens, act):
    d_in, d_out = 384, 200
    x, w = random_operand(tokens, d_in, 1, spread=0), random_operand(d_out, d_in, 2, True, spread=0)
    bias, r = normal(1, d_out, 3, dtype)[0], normal(tokens, d_out, 4, dtype, 5)
    y, held = torch.empty((tokens, d_out), dtype=TYPES[dtype], device="cuda"), None
    held = api.checkpoint_like(y)
    api.linear_fp8_forward(x, w, y, bias=bias, activation=act, residual=r, checkpoint=held)
    soft = {"none": lambda z: z, "relu": lambda z: np.maximum(z, 0), "silu": lambda z: z / (1 + np.exp(-z)),
            "gelu": lambda z: z * np.vectorize(lambda v: 0.5 * math.erfc(-v / math.sqrt(2)))(z)}[act]
    # no slope is over 1.13; gelu's erf is good to 1.5e-7 of z
    product_error(f64(y), value(x), value(w), dtype, lambda z: soft(z + f64(bias)) + f64(r), 1.13, what=act)
    z = value(x) @ value(w).T + f64(bias)
    step = np.exp2(f64(held[1]) - 127).repeat(32, axis=1)[:, :d_out]
    size = np.sqrt((value(x) ** 2) @ (value(w) ** 2).T)
    kept = f64(held[0]) * step
    assert (np.abs(kept - z) <= 0.5 * step + 2.0**-10 * np.sqrt(6) * size).all()
    same = r.clone()
    api.linear_fp8_forward(x, w, same, bias=bias, activation=act, residual=same)
    assert torch.equal(same, y)


# a bias, an activation, its checkpoint and a residual in place, rows of which are wider, on the large tiles (cut and whole) and
# on products whose k is split
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(4096 + 77, 290, 4096 + 130), (4096, 2048, 4096), (2045, 1001, 5000), (600, 2049, 5000),
                                               (1300, 1291, 777), (257, 6000, 129), (130, 6000, 4100), (64, 17025, 40), (1, 300, 8200)])
def test_epilogue_of_every_tile(dtype, tokens, d_in, d_out):
    x, w = random_operand(tokens, d_in, 1, spread=0), random_operand(d_out, d_in, 2, True, spread=0)
    bias, y = normal(1, d_out, 3, dtype)[0], normal(tokens, d_out, 4, dtype, 5)
    behind = y.as_strided((tokens, 5), (d_out + 5, 1), d_out)
    kept, r, held = behind.clone(), f64(y), api.checkpoint_like(y)
    api.linear_fp8_forward(x, w, y, bias=bias, activation="silu", residual=y, checkpoint=held)
    a, b = value(x), value(w)
    silu = lambda z: z * 0.5 * (1 + np.tanh(z / 2))
    product_error(f64(y), a, b, dtype, lambda z: silu(z + f64(bias)) + r, 1.13, what=f"{dtype} {tokens} {d_in}->{d_out}")
    assert torch.equal(behind, kept)
    z, size = matmul64(a, b) + f64(bias), np.sqrt(matmul64(a * a, b * b))
    step = np.exp2(f64(held[1]) - 127).repeat(32, axis=1)[:, :d_out]
    # half a step, and what the product itself may be off by (no more than 2^-10 of an instruction's 64 products)
    assert (np.abs(f64(held[0]) * step - z) <= 0.5 * step + 2.0**-10 * np.sqrt(-(-d_in // 64)) * size).all()


def test_row_scales_of_both_operands_and_their_extremes():
    # blocks of very different sizes whose products meet: 2^-100 of one with 2^100 of the other; scales 0 and 254
    tokens, d_in, d_out = 130, 520, 140
    for dtype in TYPES:
        x, w = random_operand(tokens, d_in, 1), random_operand(d_out, d_in, 2)
        x[1][:, 1] -= 90
        w[1][:, 1] += 90
        x[1][:, 2], w[1][:, 2] = 0, 254
        x[1][:, 3], w[1][:, 3] = 200, 50
        y = torch.empty((tokens, d_out), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
        api.linear_fp8_forward(x, w, y)
        product_error(f64(y), value(x), value(w), "f32" if dtype == "f32" else "bf16")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 100, 300])
def test_blocks_that_are_not_finite(dtype, tokens):
    x, w = random_operand(tokens, 300, 1), random_operand(200, 300, 2, True)
    x[1][1, 1] = 255
    x[0].view(torch.uint8)[1, 128:256] = 0x7F
    x[0].view(torch.uint8)[2, 299] = 0xFF
    y = torch.empty((tokens, 200), dtype=TYPES[dtype], device="cuda")
    api.linear_fp8_forward(x, w, y)
    nan = y.isnan().cpu()
    assert nan[1:3].all() and nan.sum() == 400
    # the weights' second tile
    w[1][1, 2] = 255
    api.linear_fp8_forward(x, w, y)
    assert y.isnan().cpu()[:, 128:].all() and not y.isnan().cpu()[0, :128].any()


def test_results_repeat_to_the_bit():
    for shape in ((300, 4096, 257), (1000, 1024, 1024), (7, 4096, 512)):
        first = forward(*shape, "bf16")
        assert torch.equal(first, forward(*shape, "bf16"))


SLOPES = {
    "none": lambda z: np.ones_like(z), "relu": lambda z: (z > 0).astype(float),
    "gelu": lambda z: np.vectorize(lambda v: 0.5 * math.erfc(-v / math.sqrt(2)))(z) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi),
    "silu": lambda z: (lambda s: s * (1 + z * (1 - s)))(1 / (1 + np.exp(-z))),
}


def backward(tokens, d_in, d_out, dtype, act="none", wanted="dx dw db", add=False, wider=0, seed=0):
    wanted = wanted.split()
    T = TYPES[dtype]
    dy = normal(tokens, d_out, seed, dtype, wider)
    x, w = random_operand(d_in, tokens, seed + 1, pad=1), random_operand(d_in, d_out, seed + 2, True, pad=1)
    more = normal(tokens, d_in, seed + 3, dtype) if add else None
    held, dz = None, f64(dy)
    if act != "none":
        z = normal(tokens, d_out, seed + 4, "f32")
        held = api.act8_quantize(z, *api.checkpoint_like(z))
        dz = dz * SLOPES[act](f64(api.act8_dequantize(*held, torch.empty_like(z))))
    out = {"dx": torch.empty(tokens, d_in, dtype=T, device="cuda"), "dw": torch.empty(d_out, d_in, dtype=T, device="cuda"),
           "db": torch.empty(d_out, dtype=T, device="cuda")}
    got = {k: v if k in wanted else None for k, v in out.items()}
    api.linear_fp8_backward(dy, x if "dw" in wanted else None, w if "dx" in wanted else None, **got, activation=act,
                            checkpoint=held, add=more)
    what = f"{dtype} {tokens} {d_in}->{d_out} {act}"
    # behind an activation a float32 dz lies within 2^-20 of the float64 one (relu's is exact), which may be the next code
    # for a value near the middle between two: an eighth of the value at most, of two values of an output at most
    flips = 0.0 if act in ("none", "relu") else 0.25
    if "dx" in wanted:
        a, b = decode(*encode(dz)), value(w)
        near = flips * np.abs(a).max() * np.abs(b).max()
        check(f64(got["dx"]), a, b, dtype, near, f64(more) if add else 0.0, what + " dx")
    if "dw" in wanted:
        a, b = decode(*encode(dz.T)), value(x)
        check(f64(got["dw"]), a, b, dtype, flips * np.abs(a).max() * np.abs(b).max(), 0.0, what + " dw")
    if "db" in wanted:
        want, size = dz.sum(axis=0), np.abs(dz).sum(axis=0)
        # (a sum of terms that are each good to 2^-20, in a tree)
        assert (np.abs(f64(got["db"]) - want) <= UNIT[dtype] * 1.01 * np.abs(want) + 2.0**-19 * size).all(), what
    return got


def check(got, a, b, dtype, near, more, what):
    if near == 0:
        product_error(got, a, b, dtype, more, what=what)
        return
    want = a @ b.T + more
    size = np.sqrt((a * a) @ (b * b).T)
    bound = UNIT[dtype] * 1.01 * np.abs(want) + 2.0**-10 * np.sqrt(-(-a.shape[1] // 64)) * size + near
    assert (np.abs(got - want) <= bound).all(), what
    # few values flip: over all outputs that is little
    assert np.linalg.norm(got - want) <= (0.6 * UNIT[dtype] + 1e-3) * np.linalg.norm(want), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(1, 1, 1), (1, 64, 130), (7, 33, 5), (64, 128, 128), (65, 257, 129), (130, 64, 1000),
                                               (1001, 130, 77), (2100, 96, 200), (300, 771, 513)])
def test_gradients(dtype, tokens, d_in, d_out):
    backward(tokens, d_in, d_out, dtype, add=tokens % 2 == 0, wider=tokens % 3)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("tokens,d_in,d_out", [(3, 70, 45), (300, 200, 264), (1000, 512, 384)])
def test_gradients_through_activations(act, tokens, d_in, d_out):
    for dtype in ("bf16", "f16"):
        backward(tokens, d_in, d_out, dtype, act, add=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(1, 64, 130), (45, 1030, 700), (257, 640, 385), (700, 2100, 770), (2045, 1024, 1001),
                                               (4096, 300, 2050)])
def test_gradients_in_wider_rows_and_in_place(dtype, tokens, d_in, d_out):
    """dx over its add and dw in wider rows, at odd distances: the same bits as apart, and nothing behind the rows."""
    dy = normal(tokens, d_out, 1, dtype, 3)
    x, w = random_operand(d_in, tokens, 2, pad=1), random_operand(d_in, d_out, 3, True, pad=1)
    z = normal(tokens, d_out, 4, "f32")
    ck = api.act8_quantize(z, *api.checkpoint_like(z))
    add = normal(tokens, d_in, 5, dtype)
    T = TYPES[dtype]
    plain = api.linear_fp8_backward(dy, x, w, dx=torch.empty(tokens, d_in, dtype=T, device="cuda"),
                                    dw=torch.empty(d_out, d_in, dtype=T, device="cuda"),
                                    db=torch.empty(d_out, dtype=T, device="cuda"), activation="silu", checkpoint=ck, add=add)
    dz = f64(dy) * SLOPES["silu"](f64(api.act8_dequantize(*ck, torch.empty_like(z))))
    for got, of, other, more in ((plain[0], dz, w, f64(add)), (plain[1], dz.T, x, 0.0)):
        a, b = decode(*encode(of)), value(other)
        check(f64(got), a, b, dtype, 0.25 * np.abs(a).max() * np.abs(b).max(), more, f"{dtype} {tokens} {d_in}->{d_out}")
    wide = torch.full((tokens, d_in + 3), 7.0, dtype=T, device="cuda"), torch.full((d_out, d_in + 5), 7.0, dtype=T, device="cuda")
    dx, dw = (t[:, :d_in] for t in wide)
    dx.copy_(add)
    db = torch.empty(d_out, dtype=T, device="cuda")
    api.linear_fp8_backward(dy, x, w, dx=dx, dw=dw, db=db, activation="silu", checkpoint=ck, add=dx)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), plain))
    assert all((t[:, d_in:] == 7).all() for t in wide)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("tokens", [6, 200, 1100])
def test_a_gradient_that_is_not_finite_stays_in_its_row_and_column(dtype, bad, tokens):
    d_in, d_out = 260, 300
    dy = normal(tokens, d_out, 1, dtype)
    dy[5, 7] = bad
    x, w = random_operand(d_in, tokens, 2, spread=0), random_operand(d_in, d_out, 3, True, spread=0)
    T = TYPES[dtype]
    dx, dw, db = api.linear_fp8_backward(dy, x, w, dx=torch.empty(tokens, d_in, dtype=T, device="cuda"),
                                         dw=torch.empty(d_out, d_in, dtype=T, device="cuda"),
                                         db=torch.empty(d_out, dtype=T, device="cuda"))
    for t, row in ((dx, 5), (dw, 7)):
        assert t[row].isnan().all() and t.isnan().sum() == d_in
    assert not db[7].isfinite() and db.isfinite().sum() == d_out - 1


@pytest.mark.parametrize("wanted", ["dx", "dw", "db", "dx dw", "dx db", "dw db"])
def test_some_gradients(wanted):
    every = backward(200, 136, 260, "bf16", "gelu")
    some = backward(200, 136, 260, "bf16", "gelu", wanted)
    for k in wanted.split():
        assert torch.equal(some[k], every[k])


def test_no_tokens():
    for d_in, d_out in ((40, 30), (200, 300)):
        dy = torch.empty(0, d_out, dtype=torch.bfloat16, device="cuda")
        w = random_operand(d_in, d_out, 1, True)
        x = api.fp8_like(torch.empty(0, d_in, device="cuda"), columns=True)
        dw, db = torch.full((d_out, d_in), 3.0, device="cuda").bfloat16(), torch.full((d_out,), 3.0, device="cuda").bfloat16()
        api.linear_fp8_backward(dy, x, w, dx=torch.empty(0, d_in, dtype=dy.dtype, device="cuda"), dw=dw, db=db)
        assert not dw.any() and not db.any()
        api.linear_fp8_forward(api.fp8_like(torch.empty(0, d_out, device="cuda")), w, torch.empty(0, d_in, dtype=dy.dtype, device="cuda"))


def test_gradient_against_differences():
    """The loss sum(y dy) along a change of one operand that the format holds exactly: y is linear in it."""
    tokens, d_in, d_out = 96, 256, 160
    g = torch.Generator(device="cuda").manual_seed(4)
    # whole numbers up to 15, with one 448 in each block so that every step is 1: sums and differences are exact codes
    def whole(rows, n):
        v = torch.randint(-7, 8, (rows, n), generator=g, device="cuda").float()
        v[:, ::128] = 448.0
        return v
    x, w, dy = whole(tokens, d_in), whole(d_out, d_in), torch.randint(-7, 8, (tokens, d_out), generator=g, device="cuda").float()
    dy[:, ::128] = 448.0
    dy[::96, :] = 448.0
    def run(x, w):
        x8, w8 = api.fp8_like(x), api.fp8_like(w)
        api.fp8_quantize(x, x8), api.fp8_quantize(w, w8)
        return float((api.linear_fp8_forward(x8, w8, torch.empty_like(dy)).double() * dy.double()).sum())
    x8t, w8t = api.fp8_like(x, columns=True), api.fp8_like(w, columns=True)
    api.fp8_quantize(x, columns=x8t), api.fp8_quantize(w, columns=w8t)
    dx, dw, _ = api.linear_fp8_backward(dy, x8t, w8t, dx=torch.empty_like(x), dw=torch.empty_like(w))
    for grad, of in ((dx, "x"), (dw, "w")):
        d = torch.randint(-7, 8, grad.shape, generator=g, device="cuda").float()
        d[:, ::128] = 0
        base = x if of == "x" else w
        up, down = (run(base + s * d, w) if of == "x" else run(x, base + s * d) for s in (1, -1))
        slope = float((grad.double() * d.double()).sum())
        # float32 sums on all sides: 2^-24 of terms of the loss's own parts
        scale = float(grad.double().norm() * d.double().norm())
        assert abs((up - down) / 2 - slope) <= 1e-4 * scale + 2.0**-20 * abs(up)


@pytest.mark.parametrize("tokens", [1, 77, 300])
def test_norm_product_and_training_together(tokens):
    """The chain as a decoder's layer runs it: norm to 8 bits, product, and the gradients back through both."""
    d, d_out, T = 512, 384, torch.bfloat16
    x, r = normal(tokens, d, 1, "bf16"), normal(tokens, d, 2, "bf16")
    nw = 1 + 0.1 * torch.randn(d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    w = (normal(d_out, d, 4, "f32") / math.sqrt(d)).to(T)
    w8, w8t = api.fp8_like(w, tiles=True), api.fp8_like(w, columns=True, tiles=True)
    api.fp8_quantize(w, w8, columns=w8t)
    y8, h, u, rstd = api.fp8_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(tokens, device="cuda")
    api.rms_norm_forward(x, nw, h, residual=r, summed=u, rstd=rstd, y8=y8)
    out = torch.empty(tokens, d_out, dtype=T, device="cuda")
    z8 = api.checkpoint_like(out)
    api.linear_fp8_forward(y8, w8, out, activation="silu", checkpoint=z8)
    product_error(f64(out), value(y8), value(w8), "bf16", lambda z: z / (1 + np.exp(-z)), 1.1)
    h8t = api.fp8_like(h, columns=True)
    api.fp8_quantize(h, columns=h8t)
    dy = normal(tokens, d_out, 5, "bf16")
    dh, dw, db = torch.empty_like(h), torch.empty_like(w), torch.empty(d_out, dtype=T, device="cuda")
    api.linear_fp8_backward(dy, h8t, w8t, dx=dh, dw=dw, db=db, activation="silu", checkpoint=z8)
    dx, dnw = api.rms_norm_backward(dh, u, nw, rstd, torch.empty_like(x), torch.empty_like(nw), add=r)
    # the whole against the formulas in 64 bits without any 8-bit rounding: e4m3 is off by 2^-4 of a value at most, 0.026 of
    # the norm over all, the int8 pre-activation by less; four of them in a chain stay under a tenth
    u64 = f64(u)
    s64 = 1 / np.sqrt((u64 * u64).mean(axis=1, keepdims=True) + 1e-6)
    h64 = u64 * s64 * f64(nw)
    z64 = h64 @ f64(w).T
    dz = f64(dy) * SLOPES["silu"](z64)
    gw = (dz @ f64(w)) * f64(nw)
    xh = u64 * s64
    want = {"dx": s64 * (gw - xh * (gw * xh).mean(axis=1, keepdims=True)) + f64(r), "dw": dz.T @ h64, "db": dz.sum(axis=0),
            "dnw": ((dz @ f64(w)) * xh).sum(axis=0)}
    for k, got in (("dx", dx), ("dw", dw), ("db", db), ("dnw", dnw)):
        assert np.linalg.norm(f64(got) - want[k]) <= 0.1 * np.linalg.norm(want[k]), k


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed with eager work between, against the eager results."""
    tokens, d, d_out = 200, 256, 300
    x, w = normal(tokens, d, 1, "bf16"), normal(d_out, d, 2, "bf16")
    nw = torch.ones(d, device="cuda")
    dy = normal(tokens, d_out, 3, "bf16")

    def make():
        return dict(x8=api.fp8_like(x), xt=api.fp8_like(x, columns=True), w8=api.fp8_like(w, tiles=True),
                    wt=api.fp8_like(w, columns=True, tiles=True), h=torch.empty_like(x), rstd=torch.empty(tokens, device="cuda"),
                    y=torch.empty_like(dy), dx=torch.empty_like(x), dw=torch.empty_like(w), dnw=torch.empty_like(nw),
                    db=torch.empty(d_out, dtype=x.dtype, device="cuda"), du=torch.empty_like(x))

    def go(s):
        api.rms_norm_forward(x, nw, s["h"], rstd=s["rstd"], y8=s["x8"])
        api.fp8_quantize(s["h"], columns=s["xt"])
        api.fp8_quantize(w, s["w8"], columns=s["wt"])
        api.linear_fp8_forward(s["x8"], s["w8"], s["y"])
        api.linear_fp8_backward(dy, s["xt"], s["wt"], dx=s["dx"], dw=s["dw"], db=s["db"])
        api.rms_norm_backward(s["dx"], x, nw, s["rstd"], s["du"], s["dnw"])

    eager, held = make(), make()
    go(held)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        go(held)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(held)
    for turn in range(4):
        x.copy_(normal(tokens, d, 10 + turn, "bf16"))
        dy.copy_(normal(tokens, d_out, 20 + turn, "bf16"))
        graph.replay()
        go(eager)
        torch.cuda.synchronize()
        for k in ("y", "dx", "dw", "db", "du", "dnw"):
            assert torch.equal(held[k], eager[k]), (turn, k)
