"""RMS norm of rows whose mean square, or its root's inverse, is no float32 number: y and its 8-bit form are the definition's."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import TYPES, f64, room
from tests._helpers import assert_close
from tests.test_gpu_rms_norm import check_fp8

pytestmark = pytest.mark.gpu


# the rows' root mean square as a power of two, and eps: 2^-140 and 2^-131 leave no float32 rstd, 2^127 a subnormal one; eps that
# counts next to the squares; ordinary rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power,eps", [(-140, 0.0), (-131, 0.0), (-127, 0.0), (-100, 0.0), (-57, 2.0**-114), (-50, 2.0**-101), (0, 0.0),
                                       (0, 1e-6), (64, 1e-6), (126.9, 0.0)])
@pytest.mark.parametrize("n", [7, 700, 769, 9000])
def test_rows_of_any_size(dtype, power, eps, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    rows = 5
    # 0.5 to 1 in size, so that none is past the type's largest number
    x = torch.rand(rows, n, generator=g, device="cuda", dtype=torch.float64) / 2 + 0.5
    x = x * torch.where(torch.rand(rows, n, generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** (power + 1)
    x = x.float().to(TYPES[dtype])
    if dtype == "bf16" and power == -140:
        x = x.clamp(min=2.0**-133)  # (its smallest number; 2^-140 would be zero)
    w = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
    y, summed, rstd, y8 = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), room(rows, n)
    held = api.checkpoint_like(x)
    api.rms_norm_forward(x, w, y, summed=summed, rstd=rstd, checkpoint=held, y8=y8, eps=eps)
    u = f64(x)
    r = 1 / np.sqrt((u * u).mean(axis=1, keepdims=True) + eps)
    assert_close(f64(y), u * r * f64(w), dtype, f"2^{power}")
    check_fp8(y8, u * r * f64(w))
    # what else leaves with it is of u as it came
    assert torch.equal(summed, x)
    alone = api.act8_quantize(x, *api.checkpoint_like(x))
    assert torch.equal(alone[0], held[0]) and torch.equal(alone[1], held[1])
    # rstd to 2^-20, or to a step of the subnormal numbers, or infinite past the largest
    got, want = f64(rstd), r[:, 0]
    past = want >= 2.0**128
    assert np.isinf(got[past]).all()
    assert (np.abs(got - want)[~past] <= 2.0**-20 * want[~past] + 2.0**-149).all()


@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_an_infinity_is_nan_and_the_rest_of_its_row_zero(eps):
    x = torch.ones(3, 300, device="cuda")
    x[1, 7] = float("inf")
    y = api.rms_norm_forward(x, torch.ones(300, device="cuda"), torch.empty_like(x), eps=eps)
    assert y[1, 7].isnan() and y[1].isnan().sum() == 1 and y[1].nan_to_num().count_nonzero() == 0
    assert (y[[0, 2]] - 1).abs().max() <= 1e-6


@pytest.mark.parametrize("most,least", [(2.0**100, 2.0**-20), (2.0**-60, 2.0**-130), (2.0**-110, 2.0**-145)])
def test_small_values_next_to_large_ones_keep_their_bits(most, least):
    x = torch.full((2, 300), least, device="cuda")
    x[0, ::100], x[1, 299] = most, -most
    y = api.rms_norm_forward(x, torch.ones(300, device="cuda"), torch.empty_like(x), eps=0.0)
    u = f64(x)
    want = u / np.sqrt((u * u).mean(axis=1, keepdims=True))
    # five roundings, or half a step of the subnormal numbers
    assert (np.abs(f64(y) - want) <= 2.0**-21 * np.abs(want) + 2.0**-149).all()
