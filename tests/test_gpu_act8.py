"""8-bit checkpoints against the format's definition in 64 bits: codes, scale bytes and values bit for bit."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def reference(x64: np.ndarray):
    """(codes, scale bytes, values) of float64 rows."""
    rows, n = x64.shape
    blocks = -(-n // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :n] = x64
    v = v.reshape(rows, blocks, 32)
    top = np.abs(v).max(axis=2)  # (NaN if there is one)
    fine = np.isfinite(top)
    m, k = np.frexp(np.where(fine, top, 1.0))
    e = np.where(m <= 127 / 128, k - 7, k - 6)
    e = np.maximum(np.where(top == 0, -127, e), -127)
    codes = np.where(fine[:, :, None], np.rint(np.where(fine[:, :, None], v, 0.0) * np.exp2(-e.astype(float))[:, :, None]), 0.0)
    values = np.where(fine[:, :, None], codes * np.exp2(e.astype(float))[:, :, None], np.nan)
    scales = np.where(fine, e + 127, 255).astype(np.uint8)
    flat = lambda a: a.reshape(rows, blocks * 32)[:, :n]  # noqa: E731
    return flat(codes).astype(np.int8), scales, flat(values)


def check(x: torch.Tensor):
    codes, scales = api.checkpoint_like(x)
    codes.fill_(99), scales.fill_(99)
    api.act8_quantize(x, codes, scales)
    want_codes, want_scales, want = reference(x.double().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    for dtype in TYPES.values():
        out = torch.empty(x.shape, dtype=dtype, device="cuda")
        api.act8_dequantize(codes, scales, out)
        with np.errstate(over="ignore"):
            rounded = torch.from_numpy(want).float().to(dtype)  # (code * 2^e is a float32)
        assert torch.equal(out.cpu().isnan(), rounded.isnan())
        assert torch.equal(torch.nan_to_num(out.cpu(), nan=0.0), torch.nan_to_num(rounded, nan=0.0)), dtype


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 7), (3, 8), (5, 31), (2, 32), (7, 33), (128, 256), (19, 769), (1, 4096),
                                    (513, 1000), (3, 16385), (70001, 3), (300, 4096)])
def test_definition(dtype, rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows * 31 + n)
    x = torch.randn(rows, n, generator=g, device="cuda") * torch.exp2(
        torch.randint(-6, 7, (rows, 1), generator=g, device="cuda").float())
    check(x.to(TYPES[dtype]))


def test_ties_and_limits_of_the_range():
    # every bfloat16 number, each in a block of its own with smaller ones; blocks on both sides of 127 * 2^e
    bits = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).cuda()
    big = torch.zeros(1 << 16, 32, dtype=torch.bfloat16, device="cuda")
    big[:, 5] = x
    big[:, 9] = x / 3
    big[:, 31] = -x / 128
    check(big)
    check(x.view(64, 1024).contiguous())
    edge = torch.tensor([127.0, 127.00001, 126.99999, 127.5, 128.0, 63.5, 2.0**-140, 2.0**-121 * 127, 3.4e38], device="cuda")
    rows = torch.zeros(edge.numel(), 40, device="cuda")
    rows[:, 0] = edge
    rows[:, 1] = 0.5
    rows[:, 2] = 1.5
    rows[:, 3] = -2.5
    check(rows)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_block_that_is_not_finite_is_nan_and_alone(bad):
    x = torch.randn(4, 100, device="cuda")
    x[1, 40] = bad
    x[3, 99] = bad
    check(x)
    codes, scales = api.checkpoint_like(x)
    api.act8_quantize(x, codes, scales)
    out = api.act8_dequantize(codes, scales, torch.empty_like(x))
    nan = out.isnan().cpu()
    assert nan[1, 32:64].all() and nan[3, 96:].all() and nan.sum() == 36


def test_slices_of_wider_rows_and_odd_addresses():
    wide = torch.randn(37, 301, device="cuda").to(torch.bfloat16)
    for part in (wide[:, :256], wide[:, 1:200], wide[3:, 45:], wide.view(-1)[1 : 1 + 36 * 301].view(36, 301)):
        check(part)
    codes, scales = api.checkpoint_like(wide[:, :77])
    api.act8_quantize(wide[:, :77].contiguous(), codes, scales)
    out = torch.full((37, 90), 7.0, device="cuda")
    api.act8_dequantize(codes, scales, out[:, 5:82])
    want = reference(wide[:, :77].double().cpu().numpy())[2]
    assert np.array_equal(out[:, 5:82].double().cpu().numpy(), want)
    assert (out[:, :5] == 7).all() and (out[:, 82:] == 7).all()


def test_no_rows_and_other_streams():
    x = torch.empty(0, 64, device="cuda")
    codes, scales = api.checkpoint_like(x)
    api.act8_quantize(x, codes, scales)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = torch.randn(64, 96, device="cuda")
        check(y)
    s.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
def test_finite_values_come_back_finite(dtype):
    """Also those whose code times the step is the power of two past the type's largest number."""
    most = torch.finfo(TYPES[dtype]).max
    parts = torch.tensor([1.0, 0.998, 0.9955, 0.99, 0.5], dtype=torch.float64) * most
    x = torch.zeros(10, 40, dtype=TYPES[dtype], device="cuda")
    x[:, 3] = torch.cat([parts, -parts]).to(TYPES[dtype]).cuda()
    x[:, 20] = x[:, 3] / 3
    assert x.isfinite().all()
    codes, scales = api.act8_quantize(x, *api.checkpoint_like(x))
    out = api.act8_dequantize(codes, scales, torch.empty_like(x))
    assert out.isfinite().all()
    half = torch.exp2(scales.double() - 128).repeat_interleave(32, dim=1)[:, :40]
    assert ((out.double() - x.double()).abs() <= half).all()
    # numbers that float16 does not have are infinities there, not its largest number
    wide = torch.tensor([[1e6, -66560.0, 65536.0 * 1.5, 1.0]], device="cuda")
    back = api.act8_dequantize(*api.act8_quantize(wide, *api.checkpoint_like(wide)), torch.empty_like(wide, dtype=torch.float16))
    assert back[0, :3].isinf().all()


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_slope_at_the_largest_numbers(name):
    eye = torch.eye(32, device="cuda")
    for value in (3.4e38, -3.4e38):
        z = torch.full((1, 32), value, device="cuda")
        held = api.act8_quantize(z, *api.checkpoint_like(z))
        dx = api.linear_backward(torch.ones_like(z), None, eye, dx=torch.empty_like(z), activation=name, checkpoint=held)[0]
        assert torch.equal(dx, torch.full_like(dx, float(value > 0)))
