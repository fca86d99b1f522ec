"""dW and dx of one call, which share a launch where that takes less time: sizes on both sides of that rule, either
product with the longer k, ragged edges, slices and shapes whose rows are no whole chunks (two launches), against float64 like
the products alone; and the same bits on every call."""

import pytest
import torch

from paper_2511_01385_amd import api
from tests.test_gpu_linear import TYPES, backward, tensors

pytestmark = pytest.mark.gpu

SIZES = [(1021, 1024, 768), (500, 256, 512), (513, 776, 1000), (131, 512, 640), (300, 640, 2048), (72, 2048, 1024), (2045, 2048, 2048),
         (1500, 1280, 2560), (900, 767, 768), (900, 768, 767), (17, 64, 64), (1, 256, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", SIZES)
def test_sizes(dtype, tokens, d_in, d_out):
    backward(tokens, d_in, d_out, dtype, "gelu", seed=tokens)
    backward(tokens, d_in, d_out, dtype, add=False, seed=tokens + 1)
    backward(tokens, d_in, d_out, dtype, "silu", pad=64, seed=tokens + 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", SIZES[:6])
def test_repeats_and_each_alone(dtype, tokens, d_in, d_out):
    """Calls repeat to the bit.  A gradient asked for alone is the same sum, in an order that its own plan may split."""
    x, w, _, _, dy, _ = tensors(tokens, d_in, d_out, dtype, 3)
    runs = []
    for which in ("both", "both", "alone"):
        dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
        if which == "both":
            api.linear_backward(dy, x, w, dx=dx, dw=dw)
        else:
            api.linear_backward(dy, None, w, dx=dx)
            api.linear_backward(dy, x, None, dw=dw)
        runs.append((dx, dw))
    for a, b, alone in zip(*runs):
        assert torch.equal(a, b)
        # one step of the storage type apart (2^-7 of a bf16 value, 2^-10 of an f16 one), or float32 sums of k terms in another order
        scale = float(alone.float().abs().max())
        step = {torch.bfloat16: 2.0**-7, torch.float16: 2.0**-10, torch.float32: 2.0**-17}[alone.dtype]
        assert float((a.float() - alone.float()).abs().max()) <= step * scale


def test_add_in_place_while_dw_is_made():
    x, w, _, _, dy, _ = tensors(500, 256, 512, "f32", 4)
    add = torch.randn(500, 256, device="cuda")
    want = api.linear_backward(dy, x, w, dx=torch.empty_like(x), dw=torch.empty_like(w), add=add)
    got = api.linear_backward(dy, x, w, dx=add, dw=torch.empty_like(w), add=add)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
