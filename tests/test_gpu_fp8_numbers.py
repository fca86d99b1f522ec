"""8-bit floating point over whole ranges of numbers: every code with every scale byte, every float16 number, every exponent of
float32, against the definition in 64 bits."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import TYPES, decode, encode, f64, room
from tests.test_gpu_fp8 import check, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
def test_every_code_with_every_scale_byte(dtype):
    """Rounded once to the type: bfloat16 has no room below 2^-133 for the smallest codes of the smallest scales.  The power of
    two past the type's largest number is that number, whichever code and byte make it."""
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 2))
    held = room(256, 256)
    for to, a in zip(held, (codes, scales)):
        to.view(torch.uint8).copy_(torch.from_numpy(a))
    out = api.fp8_dequantize(held, torch.empty(256, 256, dtype=TYPES[dtype], device="cuda")).cpu()
    wide = torch.from_numpy(decode(np.where(codes & 127 == 127, 0, codes), scales))
    wide = torch.where(torch.from_numpy(codes & 127 == 127), torch.nan, wide)
    most = torch.finfo(TYPES[dtype]).max
    wide = torch.where(wide.abs() == (65536.0 if dtype == "f16" else 2.0**128), torch.sign(wide) * most, wide)
    want = wide.float().to(TYPES[dtype])  # (the values are float32 numbers, or past them all)
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.equal(out.nan_to_num(nan=0.0, posinf=float("inf"), neginf=-float("inf")),
                       want.nan_to_num(nan=0.0, posinf=float("inf"), neginf=-float("inf")))


def test_every_float16_number():
    x = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16).view(torch.float16).cuda()
    big = torch.zeros(1 << 16, 128, dtype=torch.float16, device="cuda")
    big[:, 5] = x
    big[:, 9] = x / 3
    big[:, 77] = -x / 200
    big[:, 127] = x / 7000
    held = room(1 << 16, 128)
    api.fp8_quantize(big, held)
    same(held, encode(f64(big)))
    check(x.view(512, 128).contiguous())
    # those that are finite, whose blocks along the columns then are too
    check(x[x.isfinite()][: 480 * 130].view(480, 130).contiguous())


@pytest.mark.parametrize("tiles", [False, True])
def test_every_exponent_of_float32(tiles):
    g = torch.Generator(device="cuda").manual_seed(1)
    mantissa = torch.rand(256, 260, generator=g, device="cuda") + 1
    sign = torch.where(torch.rand(256, 260, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    e = torch.arange(-149, 107, device="cuda").unsqueeze(1).double()
    # a row's values lie within 2^20 of each other
    x = (mantissa.double() * sign * torch.exp2(e + torch.randint(0, 21, (256, 260), generator=g, device="cuda"))).float()
    assert x.isfinite().all() and (x != 0).all()
    check(x, tiles)
    check(x.flip(0).t().contiguous(), tiles)
