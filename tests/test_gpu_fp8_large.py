"""Matrices of more than 2^31 values: the last rows and columns against float64, which offsets of 32 bits would miss."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import decode, encode, f64, product_error, random_operand, value
from tests._helpers import assert_close

pytestmark = pytest.mark.gpu

ROWS, N = 70001, 32768  # 2.3e9 values


@pytest.fixture(scope="module")
def x():
    g = torch.Generator(device="cuda").manual_seed(1)
    yield torch.randn(ROWS, N, generator=g, device="cuda", dtype=torch.bfloat16)
    torch.cuda.empty_cache()


def part(held, rows):
    return held[0][rows].view(torch.uint8).cpu().numpy(), held[1][rows].cpu().numpy()


def test_quantize_and_back(x):
    held, columns = api.fp8_like(x), api.fp8_like(x, columns=True)
    api.fp8_quantize(x, held, columns=columns)
    last = slice(ROWS - 130, ROWS)
    for got, want in ((part(held, last), encode(f64(x[last]))), (part(columns, slice(N - 2, N)), encode(f64(x[:, N - 2 :].t().contiguous())))):
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    del columns
    out = api.fp8_dequantize(held, torch.empty_like(x))
    assert np.array_equal(f64(out[last]), decode(*encode(f64(x[last]))))


def test_products(x):
    held = api.fp8_like(x)
    api.fp8_quantize(x, held)
    w = random_operand(80, N, 2, True, spread=0)
    y = api.linear_fp8_forward(held, w, torch.empty(ROWS, 80, dtype=torch.bfloat16, device="cuda"))
    last = slice(ROWS - 100, ROWS)
    product_error(f64(y[last]), decode(*part(held, last)), value(w), "bf16")
    del held
    # a large result, and a large operand of 16-bit gradients
    a, b = random_operand(ROWS, 48, 3, spread=0), random_operand(N, 48, 4, spread=0)
    y = api.linear_fp8_forward(a, b, torch.empty_like(x))
    product_error(f64(y[last, N - 300 :]), decode(*part(a, last)), decode(*part(b, slice(N - 300, N))), "bf16")
    wt, dx = random_operand(64, N, 5, True, spread=0), torch.empty(ROWS, 64, dtype=torch.bfloat16, device="cuda")
    api.linear_fp8_backward(x, None, wt, dx=dx)
    product_error(f64(dx[last]), decode(*encode(f64(x[last]))), value(wt), "bf16")


def test_norm(x):
    u = x.view(2 * ROWS, N // 2)
    w, rstd = torch.rand(N // 2, device="cuda") + 0.5, torch.empty(2 * ROWS, device="cuda")
    y, y8 = torch.empty_like(u), api.fp8_like(u)
    api.rms_norm_forward(u, w, y, rstd=rstd, y8=y8)
    last = slice(2 * ROWS - 50, 2 * ROWS)
    u64 = f64(u[last])
    s64 = 1 / np.sqrt((u64 * u64).mean(axis=1, keepdims=True) + 1e-6)
    want = u64 * s64 * f64(w)
    assert_close(f64(y[last]), want, "bf16")
    near = decode(*part(y8, last))
    assert (np.abs(near - want) <= 2.0**-4 * 1.001 * np.abs(want) + 2.0**-9 * np.abs(want).max()).all()
    dx = api.rms_norm_backward(y, u, w, rstd, y)[0]
    dy = want.astype(np.float32)  # (y as it was, but for its rounding: dx is linear in it)
    g = torch.from_numpy(dy).to(torch.bfloat16).double().numpy() * f64(w)
    xh = u64 * s64
    assert np.linalg.norm(f64(dx[last]) - s64 * (g - xh * (g * xh).mean(axis=1, keepdims=True))) <= 0.02 * np.linalg.norm(s64 * g)
