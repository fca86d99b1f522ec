"""The dense product with its epilogue, and its gradients, against the formulas in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._helpers import assert_close

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def tensors(tokens, d_in, d_out, dtype, seed, pad=0, shift=0):
    """x, w, bias, residual, dy, add of a layer that keeps the variance; rows `pad` longer, starting at element `shift`."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def make(rows, n, scale=1.0):
        flat = torch.randn(rows * (n + pad) + shift, generator=g, device="cuda") * scale
        return flat.to(TYPES[dtype])[shift:].view(rows, n + pad)[:, :n]

    return (make(tokens, d_in), make(d_out, d_in, 1 / math.sqrt(d_in)), make(1, d_out)[0].contiguous(), make(tokens, d_out),
            make(tokens, d_out), make(tokens, d_in))


def forward(tokens, d_in, d_out, dtype, activation="none", bias=True, residual=True, checkpoint=False, seed=0, pad=0, shift=0):
    x, w, b, r, _, _ = tensors(tokens, d_in, d_out, dtype, seed, pad, shift)
    y = torch.full((tokens, d_out + pad), 5.0, dtype=TYPES[dtype], device="cuda")
    held = api.checkpoint_like(r) if checkpoint else None
    api.linear_forward(x, w, y[:, :d_out], bias=b if bias else None, activation=activation,
                       residual=r if residual else None, checkpoint=held)
    assert (y[:, d_out:] == 5).all()
    z = x.double() @ w.double().t()
    if bias:
        z = z + b.double()
    want = act(activation, z)
    if residual:
        want = want + r.double()
    what = f"{dtype} {tokens} {d_in}->{d_out} {activation}"
    got, want = y[:, :d_out].double().cpu().numpy(), want.cpu().numpy()
    if d_out < 16:  # (the rule's rms is over a row)
        got, want = got.reshape(1, -1), want.reshape(1, -1)
    assert_close(got, want, dtype, what)
    if checkpoint:
        codes, scales = held
        values = api.act8_dequantize(codes, scales, torch.empty(tokens, d_out, device="cuda")).double()
        step = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)[:, :d_out]
        # half a step, and float32 sums
        assert ((values - z).abs() <= 0.5 * step + 2e-5 * z.pow(2).mean().sqrt()).all(), what
        # no block has a larger step than it needs, but for a maximum at the very edge
        pad_z = torch.nn.functional.pad(z.abs(), (0, -d_out % 32)).view(tokens, -1, 32).amax(dim=2)
        exp = torch.ceil(torch.log2(pad_z / 127))
        off = exp + 127 != scales.double()
        near = (torch.log2(pad_z / 127) - torch.round(torch.log2(pad_z / 127))).abs() < 1e-4
        assert not (off & ~near).any(), what


def backward(tokens, d_in, d_out, dtype, activation="none", which="xwb", add=True, seed=0, pad=0, shift=0):
    x, w, _, z, dy, a = tensors(tokens, d_in, d_out, dtype, seed, pad, shift)
    held = None
    zq = None
    if activation != "none":
        held = api.checkpoint_like(z)
        api.act8_quantize(z, *held)
        zq = api.act8_dequantize(*held, torch.empty(tokens, d_out, device="cuda")).double()
    new = lambda *s: torch.full(s, 5.0, dtype=TYPES[dtype], device="cuda")  # noqa: E731
    dx = new(tokens, d_in + pad)[:, :d_in] if "x" in which else None
    dw = new(d_out, d_in + pad)[:, :d_in] if "w" in which else None
    db = new(d_out) if "b" in which else None
    api.linear_backward(dy, x, w, dx=dx, dw=dw, db=db, activation=activation, checkpoint=held, add=a if add else None)
    dz = dy.double()
    if activation != "none":
        dz = dz * slope(activation, zq)
    # the products take dz rounded to the storage type, which spreads as one staged rounding does
    operand, staged = (dz, 0) if activation == "none" else (dz.to(TYPES[dtype]).double(), 1)
    what = f"{dtype} {tokens} {d_in}->{d_out} {activation}"

    def close(got, want, name, staged):
        assert_close(got.double().cpu().numpy().reshape(1, -1), want.cpu().numpy().reshape(1, -1), dtype, what + name, staged)

    if dx is not None:
        close(dx, operand @ w.double() + (a.double() if add else 0), " dx", staged)
    if dw is not None and tokens > 0:
        close(dw, operand.t() @ x.double(), " dw", staged)
    if db is not None and tokens > 0:
        close(db, dz.sum(dim=0), " db", 0)
    return dx, dw, db


SIZES = [(1, 64, 64), (1, 4096, 4096), (2, 1, 1), (3, 7, 5), (5, 8, 33), (16, 96, 40), (17, 769, 130), (61, 1024, 4096),
         (64, 64, 8192), (65, 200, 72), (127, 4096, 96), (128, 128, 128), (129, 136, 264), (200, 1001, 999),
         (300, 768, 768), (1000, 72, 2000), (2045, 256, 512), (4100, 64, 64), (700, 2048, 1031)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", SIZES)
def test_forward_sizes(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, seed=tokens)
    forward(tokens, d_in, d_out, dtype, "gelu", residual=False, checkpoint=True, seed=tokens + 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,d_in,d_out", SIZES)
def test_backward_sizes(dtype, tokens, d_in, d_out):
    backward(tokens, d_in, d_out, dtype, seed=tokens)
    backward(tokens, d_in, d_out, dtype, "silu", add=False, seed=tokens + 1)


@pytest.mark.parametrize("tokens,d_in,d_out", [(4096, 2048, 4096), (3000, 4096, 4104), (8200, 1000, 2048)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, "gelu", checkpoint=True)
    backward(tokens, d_in, d_out, dtype, "gelu")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
def test_forms(dtype, activation):
    for bias in (False, True):
        for residual in (False, True):
            forward(150, 320, 224, dtype, activation, bias, residual, checkpoint=residual)
            forward(9, 320, 224, dtype, activation, bias, residual, checkpoint=bias)
    for which in ("x", "w", "b", "xb", "wb"):
        backward(150, 320, 224, dtype, activation, which)
        backward(9, 320, 224, dtype, activation, which)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (64, 0), (0, 1), (8, 3), (0, 8)])
def test_strides_and_alignment(dtype, pad, shift):
    for tokens in (5, 200, 600):
        forward(tokens, 264, 520, dtype, "relu", checkpoint=True, pad=pad, shift=shift)
        backward(tokens, 264, 520, dtype, "relu", pad=pad, shift=shift)


def test_in_place():
    x, w, b, r, dy, a = tensors(300, 256, 640, "bf16", 3)
    want = api.linear_forward(x, w, torch.empty_like(r), bias=b, residual=r, activation="gelu")
    y = r.clone()
    api.linear_forward(x, w, y, bias=b, residual=y, activation="gelu")
    assert torch.equal(y, want)
    want = api.linear_backward(dy, x, w, dx=torch.empty_like(x), add=a)[0]
    dx = a.clone()
    api.linear_backward(dy, x, w, dx=dx, add=dx)
    assert torch.equal(dx, want)


def test_refusals():
    x, w, b, r, dy, a = tensors(40, 96, 160, "bf16", 3)
    y = torch.empty_like(r)
    held = api.checkpoint_like(r)
    for args, kw, err in (((x, w.half(), y), {}, TypeError), ((x, w[:, :95], y), {}, ValueError), ((x, w, y[:39]), {}, ValueError),
                          ((x, w.cpu(), y), {}, ValueError), ((x, w, y), dict(bias=b.float()), TypeError),
                          ((x, w, y), dict(bias=b[1:]), ValueError), ((x, w, y), dict(activation="tanh"), ValueError),
                          ((x, w, y), dict(residual=r[:, 1:]), ValueError), ((x, w, y), dict(checkpoint=(held[1], held[0])), TypeError),
                          ((x, w, y), dict(checkpoint=(held[0], held[1][:, :4])), ValueError), ((x, w, x[:, :160]), {}, ValueError),
                          ((x, w, w[:40, :1].expand(40, 160)), {}, ValueError), ((x.double(), w, y), {}, TypeError)):
        with pytest.raises(err):
            api.linear_forward(*args, **kw)
    for kw, err in ((dict(dx=a, activation="gelu"), ValueError), (dict(dx=a[:, :95]), ValueError), (dict(dw=w.float()), TypeError),
                    (dict(dx=a, dw=w[:, :95]), ValueError), (dict(db=b[:5]), ValueError), (dict(dx=dy[:, :96]), api.RdfftError)):
        with pytest.raises(err):
            api.linear_backward(dy, x, w, **kw)
    with pytest.raises(ValueError):
        api.linear_backward(dy, None, w, dw=torch.empty_like(w))


def test_no_tokens():
    x, w, b, r, dy, a = tensors(0, 96, 160, "bf16", 3)
    api.linear_forward(x, w, torch.empty_like(r), bias=b)
    dw, db = torch.full_like(w, 3), torch.full_like(b, 3)
    held = api.checkpoint_like(r)
    api.linear_backward(dy, x, w, dx=torch.empty_like(x), dw=dw, db=db, activation="gelu", checkpoint=held)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("tokens", [3, 300])
def test_values_that_are_not_finite_stay_in_their_row(tokens):
    x, w, b, r, dy, _ = tensors(tokens, 200, 72, "bf16", 5)
    x[1, 199] = float("inf")
    x[2, 0] = float("nan")
    held = api.checkpoint_like(r)
    y = api.linear_forward(x, w, torch.empty_like(r), bias=b, activation="relu", checkpoint=held)
    bad = (~y.isfinite()).any(dim=1).cpu()
    assert bad[1] and bad[2] and bad.sum() == 2
    assert y[2].isnan().all()
    assert (held[1][2] == 255).all() and (held[1][1] == 255).all() and (held[1] == 255).any(dim=1).sum() == 2
    # its gradient: NaN in the rows whose checkpoint is, and nowhere else
    dx = api.linear_backward(dy, x, w, dx=torch.empty_like(x), activation="gelu", checkpoint=held)[0]
    assert dx[1].isnan().all() and dx[2].isnan().all() and dx.isnan().any(dim=1).sum() == 2


def test_large_pre_activations():
    # far out, relu, gelu and silu are z or 0 and their slopes 1 or 0
    z = torch.tensor([-1e30, -3e4, -200.0, -40.0, 40.0, 200.0, 3e4, 1e30] * 4, device="cuda").view(1, 32)
    eye = torch.eye(32, device="cuda")
    for name in ("relu", "gelu", "silu"):
        y = api.linear_forward(z, eye, torch.empty_like(z), activation=name)
        assert torch.equal(y, z.clamp(min=0)) or (y - z.clamp(min=0)).abs().max() < 1e-12, name
    for value in (-3e4, -200.0, 200.0, 3e4):
        flat = torch.full((1, 32), value, device="cuda")
        held = api.checkpoint_like(flat)
        api.act8_quantize(flat, *held)
        dy = torch.ones_like(flat)
        for name in ("relu", "gelu", "silu"):
            dx = api.linear_backward(dy, None, eye, dx=torch.empty_like(flat), activation=name, checkpoint=held)[0]
            assert torch.equal(dx, torch.full_like(dx, float(value > 0))), (name, value)


def test_results_repeat_to_the_bit():
    for tokens in (40, 2000):
        first = backward(tokens, 768, 768, "bf16", "gelu")
        second = backward(tokens, 768, 768, "bf16", "gelu")
        assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_gradient_against_differences():
    # float32, no rounding of the operands; the gradient is taken at the checkpoint's values, so x and the bias are
    # chosen such that the pre-activation is one (integers up to 127 in every block)
    tokens, d_in, d_out = 64, 96, 160
    g = torch.Generator(device="cuda").manual_seed(11)
    z = torch.randint(-127, 128, (1, d_out), generator=g, device="cuda").float() / 32
    z[:, ::32] = 127 / 32
    x = torch.randn(tokens, d_in, generator=g, device="cuda")
    w = torch.zeros(d_out, d_in, device="cuda")
    b = z[0].contiguous()
    dy = torch.randn(tokens, d_out, generator=g, device="cuda")
    for name in ("gelu", "silu"):
        held = api.checkpoint_like(dy)
        api.linear_forward(x, w, torch.empty_like(dy), bias=b, activation=name, checkpoint=held)
        dw, db = torch.empty_like(w), torch.empty_like(b)
        api.linear_backward(dy, x, w, dw=dw, db=db, activation=name, checkpoint=held)
        h = 2.0**-7
        for grad, at in ((dw, "w"), (db, "b")):
            d = torch.randn(grad.shape, generator=g, device="cuda") * (0.1 if at == "w" else 1.0)
            loss = []
            for s in (h, -h):
                y = api.linear_forward(x, w + s * d if at == "w" else w, torch.empty_like(dy),
                                       bias=b + s * d if at == "b" else b, activation=name)
                loss.append(float((y.double() * dy.double()).sum()))
            slope_ = float((grad.double() * d.double()).sum())
            # third derivatives of order one: h^2 / 6; float32 rounding of y: 2^-24 / h
            scale = float(grad.double().norm() * d.double().norm())
            assert abs((loss[0] - loss[1]) / (2 * h) - slope_) < 1e-3 * scale, (name, at)


def test_on_another_stream_and_with_a_workspace_of_ones_own():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        forward(40, 768, 768, "bf16", "gelu", checkpoint=True)
        backward(40, 768, 768, "bf16", "gelu")
        x, w, b, r, dy, a = tensors(40, 768, 768, "bf16", 3)
        need = max(api.linear_forward_workspace(768, 768, 40, torch.bfloat16), 256)
        one = api.linear_forward(x, w, torch.empty_like(r), workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
        assert torch.equal(one, api.linear_forward(x, w, torch.empty_like(r)))
    s.synchronize()


def test_replayed_from_a_graph():
    x, w, b, r, dy, a = tensors(520, 512, 768, "bf16", 4)
    y, dx, dw, db = torch.empty_like(r), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    held = api.checkpoint_like(r)

    def step():
        api.linear_forward(x, w, y, bias=b, activation="gelu", checkpoint=held)
        api.linear_backward(dy, x, w, dx=dx, dw=dw, db=db, activation="gelu", checkpoint=held, add=a)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(k)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        dy.copy_(torch.randn(dy.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (y, dx, dw, db))), k


@pytest.mark.parametrize("dtype", TYPES)
def test_one_row_of_a_long_stride(dtype):
    """The last token of a sequence: one row, whose stride (the sequence) reaches nothing."""
    x, w, b, r, dy, a = tensors(1, 512, 96, dtype, 3)

    def last(t):
        rows = torch.zeros(1, 5000, t.shape[1], dtype=t.dtype, device="cuda")
        rows[:, -1, :] = t
        return rows[:, -1, :]

    assert last(x).stride(0) > 1 << 21
    want = api.linear_forward(x, w, torch.empty_like(r), bias=b, residual=r)
    assert torch.equal(api.linear_forward(last(x), w, last(r), bias=b, residual=last(r)), want)
    y = last(r)
    assert torch.equal(api.linear_forward(x, w, y, bias=b, residual=y.as_strided((1, 96), (96, 1))), want)
    dx, dw = api.linear_backward(dy, x, w, dx=torch.empty_like(x), dw=torch.empty_like(w), add=a)[:2]
    got = api.linear_backward(last(dy), last(x), w, dx=last(a), dw=torch.empty_like(w), add=last(a))
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


# Sizes (tokens, d_in, d_out) for the kernels that those above leave out; what the plan takes for them is named.
WHOLE = [
    (806, 5328, 16),      # y: 64 x 64, k split
    (4179, 4456, 78),     # y: 128 x 128, k split
    (12440, 712, 296),    # y: 128 x 256
    (68, 6728, 11220),    # y: 128 x 256, k split
    (133, 10720, 12632),  # y: 256 x 256, k split
    (1176, 16, 3448),     # dx: 64 x 64, k split
    (12840, 72, 16),      # dx: 64 x 64
    (12931, 208, 16),     # dx: 128 x 128
    (74, 2704, 7608),     # dx: 128 x 128, k split
    (5554, 152, 4800),    # dx: 128 x 256, k split
    (3103, 3848, 688),    # dx: 256 x 256
    (165, 10928, 8512),   # dx: 256 x 256, k split
    (7470, 2808, 72),     # dW: 128 x 128, k split
    (4884, 136, 5488),    # dW: 128 x 256, k split
    (691, 7600, 1600),    # dW: 256 x 256
    (7823, 136, 11440),   # dW: 256 x 256, k split
]
CUT = [
    (74, 1353, 16),       # y: 64 x 64, k split
    (4651, 17, 656),      # y: 128 x 128
    (2093, 10314, 72),    # y: 128 x 128, k split
    (308, 773, 11703),    # y: 128 x 256
    (65, 6309, 12344),    # y: 128 x 256, k split
    (69, 17, 1559),       # dx: 64 x 64, k split
    (584, 4925, 16),      # dx: 128 x 128
    (2314, 67, 8312),     # dx: 128 x 128, k split
    (11405, 273, 721),    # dx: 128 x 256
    (6498, 131, 4920),    # dx: 128 x 256, k split
    (1264, 17, 24),       # dW: 64 x 64, k split
    (71, 402, 7099),      # dW: 128 x 128
    (6403, 3332, 81),     # dW: 128 x 128, k split
    (61, 1001, 999), (40, 333, 8200), (33, 77, 8195),  # few tokens
]
FLOAT = [
    (8549, 1256, 16),     # y: 64 x 64, k split
    (9695, 16, 1280),     # dx: 64 x 64, k split
    (107, 531, 16),       # y: 32 x 64, cut, k split
    (11915, 17, 144),     # y: 64 x 64, cut
    (8782, 959, 16),      # y: 64 x 64, cut, k split
    (70, 19, 591),        # dx: 32 x 64, cut, k split
    (11699, 137, 18),     # dx: 64 x 64, cut
    (8523, 17, 1232),     # dx: 64 x 64, cut, k split
    (385, 19, 16),        # dW: 64 x 64, cut, k split
    (61, 1001, 999), (40, 333, 8200), (33, 77, 8195),  # few tokens, cut
]


@pytest.mark.parametrize("dtype,tokens,d_in,d_out", [(t, *s) for t in ("bf16", "f16") for s in WHOLE + CUT]
                         + [("f32", *s) for s in FLOAT])
def test_every_tile(dtype, tokens, d_in, d_out):
    forward(tokens, d_in, d_out, dtype, seed=tokens)
    forward(tokens, d_in, d_out, dtype, "gelu", checkpoint=True, seed=tokens + 1)
    for which in ("x", "w"):  # (apart: each with a plan of its own)
        backward(tokens, d_in, d_out, dtype, which=which, seed=tokens + 2)
        backward(tokens, d_in, d_out, dtype, "silu", which=which, add=False, seed=tokens + 3)
