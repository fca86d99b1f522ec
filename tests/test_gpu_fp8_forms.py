"""Forms of the 8-bit product that its operands' scales and its length along k can take: an x in tiles, and every tile with its
k in ranges.  Against float64 on the GPU, with the bounds that _fp8.product_error derives."""

import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import TYPES, UNIT, decode, encode, f64, product_error, random_operand, value

pytestmark = pytest.mark.gpu


# few tokens, whole and cut tiles; the scales' second band begins inside a tile of 64 x 128 and inside one of 256 x 256
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w_tiles", [False, True])
@pytest.mark.parametrize("tokens,d_in,d_out", [(3, 700, 200), (60, 300, 130), (100, 1001, 257), (257, 6000, 129), (1000, 640, 512),
                                               (2045, 1291, 4100)])
def test_x_in_tiles(dtype, w_tiles, tokens, d_in, d_out):
    x, w = random_operand(tokens, d_in, 1, True, pad=1, spread=1), random_operand(d_out, d_in, 2, w_tiles, pad=1, spread=1)
    x[1][0, 0] += 3  # (neighbouring tiles of one size would hide which of them a row takes)
    x[1][-1, -1] -= 3
    y = torch.empty(tokens, d_out, dtype=TYPES[dtype], device="cuda")
    api.linear_fp8_forward(x, w, y)
    product_error(f64(y), value(x), value(w), dtype, what=f"{dtype} {tokens} {d_in}->{d_out}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", [(3, 300, 200), (100, 257, 64), (300, 129, 200), (1000, 384, 520)])
def test_columns_of_x_in_tiles(dtype, tokens, d_in, d_out):
    x, w = random_operand(d_in, tokens, 1, True, pad=1, spread=1), random_operand(d_in, d_out, 2, False, pad=1, spread=1)
    x[1][-1, 0] += 3
    dy = torch.randn(tokens, d_out, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(TYPES[dtype])
    dx, dw = torch.empty(tokens, d_in, dtype=dy.dtype, device="cuda"), torch.empty(d_out, d_in, dtype=dy.dtype, device="cuda")
    api.linear_fp8_backward(dy, x, w, dx=dx, dw=dw)
    product_error(f64(dx), decode(*encode(f64(dy))), value(w), dtype, what="dx")
    product_error(f64(dw), decode(*encode(f64(dy).T)), value(x), dtype, what="dw")
    alone = api.linear_fp8_backward(dy, x, None, dw=torch.empty_like(dw))[1]
    product_error(f64(alone), decode(*encode(f64(dy).T)), value(x), dtype, what="dw alone")


def held_values(rows, n, seed, tiles):
    """An operand that fp8_quantize leaves of normal values (in rows whose padding is junk), and the float64 values it stands for."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.full((rows, -(-n // 16) * 16 + 16), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :n]
    blocks, bands = -(-n // 128), -(-rows // 128) if tiles else rows
    scales = torch.full((bands, -(-blocks // 4) * 4 + 4), 255, dtype=torch.uint8, device="cuda")[:, :blocks]
    size = torch.exp2(torch.randint(-1, 2, (1, n), generator=g, device="cuda").float())
    api.fp8_quantize(torch.randn(rows, n, generator=g, device="cuda") * size, (codes, scales))
    power = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), scales.int() - 127)
    power = power if bands == rows else power.repeat_interleave(128, dim=0)[:rows]
    return (codes, scales), codes.double() * power.repeat_interleave(128, dim=1)[:, :n]


def close(got, want, size, k, dtype, slope, what):
    """product_error's rule, on the GPU (float16 results have to be in its range)."""
    got = got.double()
    bound = (UNIT[dtype] * 1.01 + 2.0**-22) * want.abs() + slope * dropped(k, dtype) * size
    off = (got - want).abs()
    assert got.isfinite().all(), what
    assert (off <= bound + (2.0**-25 if dtype == "f16" else 0.0)).all(), what
    norm = want.norm()
    all_off = 1e-6 if dtype == "f32" else 1e-4 * max(1.0, slope * float(size.norm() / norm))
    assert off.norm() <= (0.6 * UNIT[dtype] + all_off) * norm, what


def dropped(k, dtype):
    """What a product may be off by, next to the 2-norm of its terms."""
    return 2.0**-22 * k**0.5 if dtype == "f32" else 2.0**-10 * (-(-k // 64)) ** 0.5


# A size for each tile of 16-bit results that the plan takes with k in ranges: 32 x 64, the same of four groups of waves, 64, 64 x
# 128, the same of two, 128, the same of two, 128 x 256 and 256, by the plan's own costs.  Ranges begin at a stage that is not a
# multiple of four (scales come for four stages at a time); rows, columns and the last chunk of k are cut.
# (test_every_tile of test_gpu_linear_fp8.py has them with k whole.)  float32 results have the smaller tiles, of which the plan never
# takes 32 x 64 with k in ranges.
RANGES = [(67, 8211, 20, 13), (65, 10436, 17, 14), (391, 7877, 261, 7), (196, 12312, 771, 9), (451, 13929, 386, 8), (1818, 13379, 1341, 3),
          (8210, 15662, 68, 3), (1255, 9427, 1621, 3), (1673, 13306, 2394, 3)]
RANGES_F32 = [(65, 8549, 20, 14), (649, 3345, 922, 3), (1091, 5661, 588, 5), (811, 3110, 606, 3)]


@pytest.mark.parametrize("dtype,tokens,d_in,d_out,ranges",
                         [(t, *r) for r in RANGES for t in ("bf16", "f16")] + [("f32", *r) for r in RANGES_F32])
def test_ranges_of_k_in_every_tile(dtype, tokens, d_in, d_out, ranges):
    assert api.linear_fp8_forward_workspace(d_in, d_out, tokens, TYPES[dtype]) == ranges * tokens * d_out * 4
    assert -(-(-(-d_in // 128)) // ranges) % 4 != 0 and d_in % 16 != 0
    x, a = held_values(tokens, d_in, 1, tokens % 2 == 1)
    w, b = held_values(d_out, d_in, 2, True)
    b = b.t().contiguous()
    z = a @ b
    size = ((a * a) @ (b * b)).sqrt()
    what = f"{dtype} {tokens} {d_in}->{d_out}"
    y = torch.empty(tokens, d_out, dtype=TYPES[dtype], device="cuda")
    close(api.linear_fp8_forward(x, w, y), z, size, d_in, dtype, 1.0, what)
    # with everything that the epilogue does, in place of the residual, in wider rows
    g = torch.Generator(device="cuda").manual_seed(3)
    bias = torch.randn(d_out, generator=g, device="cuda").to(y.dtype)
    wide = torch.randn(tokens, d_out + 5, generator=g, device="cuda").to(y.dtype)
    kept, place = wide.clone(), wide[:, :d_out]
    held = api.checkpoint_like(place)
    api.linear_fp8_forward(x, w, place, bias=bias, activation="silu", residual=place, checkpoint=held)
    z = z + bias.double()
    # no slope of silu is over 1.1; a sum with the residual that ends up small has roundings of its terms
    more = kept[:, :d_out].double()
    close(place, z * torch.sigmoid(z) + more, size + (2.0**-22 / dropped(d_in, dtype)) * (z.abs() + more.abs()), d_in, dtype, 1.1,
          what + " with its epilogue")
    assert torch.equal(wide[:, d_out:], kept[:, d_out:])
    step = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), held[1].int() - 127).repeat_interleave(32, dim=1)[:, :d_out]
    # (a float32 z lies within 2^-22 of itself, too)
    assert ((held[0].double() * step - z).abs() <= 0.5 * step + dropped(d_in, dtype) * size + 2.0**-22 * z.abs()).all(), what
