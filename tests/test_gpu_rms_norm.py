"""RMS norm forward and backward against the formulas in 64 bits (the comparison rule of _helpers)."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._fp8 import TABLE, TYPES, encode, f64, host, room
from tests._helpers import assert_close

pytestmark = pytest.mark.gpu

EPS = 1e-6


def hidden(rows, n, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda") + 0.3 * torch.randn(n, generator=g, device="cuda")
    return x.to(TYPES[dtype])


def check_fp8(held, y):
    """held is y's 8-bit form, of a float32 y within 2^-21 of the float64 one (three products, a sum in a tree and a root)."""
    codes, scales = host(held)
    want_codes, want_scales = encode(y)
    # the block's scale is another one only where the largest value is that near to 448 times a power of two
    power = np.exp2(want_scales.astype(float) - 127)
    top = np.abs(np.pad(y, ((0, 0), (0, -y.shape[1] % 128))).reshape(y.shape[0], -1, 128)).max(axis=2)
    near = (np.abs(top / (448 * power) - 1) < 2.0**-20) | (np.abs(top / (224 * power) - 1) < 2.0**-20)
    assert np.array_equal(scales[~near], want_scales[~near])
    fine = np.repeat(scales == want_scales, 128, axis=1)[:, : y.shape[1]]
    # a code is another one, the next, only where the value is that near to the middle between two
    off = fine & (codes != want_codes)
    q = np.abs(y) / np.repeat(power, 128, axis=1)[:, : y.shape[1]]
    lo = np.clip(np.searchsorted(TABLE, q, side="right") - 1, 0, 125)
    middle = (TABLE[lo] + TABLE[lo + 1]) / 2
    assert (np.abs(q - middle)[off] <= 2.0**-20 * middle[off]).all()
    assert (np.abs((codes & 127).astype(int) - (want_codes & 127))[off] == 1).all()


def run(rows, n, dtype, residual=False, checkpoint=False, add=False, pad=0, seed=0):
    """Forward and backward through the library, each result checked."""
    T = TYPES[dtype]
    x = hidden(rows, n + pad, seed, dtype)[:, :n]
    r = hidden(rows, n + 2 * pad, seed + 1, dtype)[:, pad : pad + n] if residual else None
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    w = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
    dy = torch.randn(rows, n + pad, generator=g, device="cuda").to(T)[:, :n]
    more = torch.randn(rows, n + pad, generator=g, device="cuda").to(T)[:, :n] if add else None
    y, summed = (torch.full((rows, n + pad), 5.0, dtype=T, device="cuda") for _ in range(2))
    rstd = torch.empty(rows, device="cuda")
    held, y8 = api.checkpoint_like(x) if checkpoint else None, room(rows, n)
    api.rms_norm_forward(x, w, y[:, :n], residual=r, summed=summed[:, :n], rstd=rstd, checkpoint=held, y8=y8, eps=EPS)
    assert (y[:, n:] == 5).all() and (summed[:, n:] == 5).all()
    what = f"{dtype} {rows}x{n}"
    # (the float32 sum of two 16-bit numbers rounds to the type as the exact one does but for ties that it makes)
    kept = (x.float() + r.float()).to(T) if residual else x
    assert torch.equal(summed[:, :n], kept)
    u = f64(kept)
    r64 = 1 / np.sqrt((u * u).mean(axis=1, keepdims=True) + EPS)
    want = u * r64 * f64(w)
    assert_close(f64(y[:, :n]), want, dtype, what + " y")
    assert np.all(np.abs(f64(rstd) / r64[:, 0] - 1) <= 2.0**-20)
    check_fp8(y8, want)
    if checkpoint:
        alone = api.act8_quantize(kept.contiguous(), *api.checkpoint_like(kept))
        assert torch.equal(alone[0], held[0]) and torch.equal(alone[1], held[1])
        u = f64(api.act8_dequantize(*held, torch.empty((rows, n), device="cuda")))

    dx = torch.full((rows, n + pad), 5.0, dtype=T, device="cuda")
    dw = torch.empty(n, device="cuda")
    api.rms_norm_backward(dy, held if checkpoint else summed[:, :n], w, rstd, dx[:, :n], dw, add=more)
    assert (dx[:, n:] == 5).all()
    s64 = f64(rstd)[:, None]
    xh, gw = u * s64, f64(dy) * f64(w)
    want = s64 * (gw - xh * (gw * xh).mean(axis=1, keepdims=True)) + (f64(more) if add else 0)
    if n > 2 or add:
        assert_close(f64(dx[:, :n]), want, dtype, what + " dx")
    else:
        # what is left of g without its part along xh may be nothing but rounding of terms of g's size
        size = s64 * np.abs(gw).max(axis=1, keepdims=True)
        assert np.all(np.abs(f64(dx[:, :n]) - want) <= 2.0**-18 * size + 2.0**-8 * np.abs(want))
    assert_close(f64(dw), (f64(dy) * xh).sum(axis=0), "f32", what + " dweight")
    alone = torch.empty_like(dx)[:, :n]
    api.rms_norm_backward(dy, held if checkpoint else summed[:, :n], w, rstd, alone, add=more)
    assert torch.equal(alone, dx[:, :n])
    return y, dx, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 2), (3, 7), (5, 8), (1, 33), (17, 256), (4, 511), (130, 513), (33, 768), (300, 769),
                                    (9, 1024), (2, 1025), (40, 2048), (7, 2049), (1, 4096), (300, 4096), (11, 4097),
                                    (5, 8192), (3, 8200), (2, 16383), (300, 16384)])
def test_widths(dtype, rows, n):
    run(rows, n, dtype, seed=n)
    run(rows, n, dtype, residual=True, checkpoint=True, add=True, seed=n + 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual,checkpoint,add,pad", [(True, False, True, 0), (False, True, False, 0), (False, False, True, 3),
                                                         (True, True, False, 5), (True, False, False, 8)])
def test_forms(dtype, residual, checkpoint, add, pad):
    for n in (260, 1027, 4099):
        run(77, n, dtype, residual, checkpoint, add, pad, seed=n)


@pytest.mark.parametrize("checkpoint", [False, True])
def test_many_rows(checkpoint):
    run(20000, 768, "bf16", residual=True, checkpoint=checkpoint, add=True)
    run(9001, 64, "f32", checkpoint=checkpoint)


def test_in_place():
    x, r = hidden(50, 1000, 1, "bf16"), hidden(50, 1000, 2, "bf16")
    w = torch.ones(1000, device="cuda")
    y, u = torch.empty_like(x), torch.empty_like(x)
    api.rms_norm_forward(x, w, y, residual=r, summed=u)
    for at_y, at_u in ((0, 1), (1, 0), (0, None), (None, 0), (None, 1)):
        pair = [x.clone(), r.clone()]
        got_y = pair[at_y] if at_y is not None else torch.empty_like(x)
        got_u = pair[at_u] if at_u is not None else torch.empty_like(x)
        api.rms_norm_forward(pair[0], w, got_y, residual=pair[1], summed=got_u)
        assert torch.equal(got_y, y) and torch.equal(got_u, u)
    rstd = torch.empty(50, device="cuda")
    api.rms_norm_forward(x, w, y, rstd=rstd)
    dw = torch.empty_like(w)
    want = api.rms_norm_backward(r, x, w, rstd, torch.empty_like(x), dw, add=u)[0]
    for place in (0, 1):
        pair = [r.clone(), u.clone()]
        api.rms_norm_backward(pair[0], x, w, rstd, pair[place], dw, add=pair[1])
        assert torch.equal(pair[place], want)


def test_zero_rows_large_values_and_no_outputs():
    w = torch.ones(700, device="cuda")
    x = torch.zeros(3, 700, device="cuda")
    y8, rstd = room(3, 700), torch.empty(3, device="cuda")
    y = api.rms_norm_forward(x, w, torch.empty_like(x), y8=y8, rstd=rstd, eps=EPS)
    assert not y.any() and not host(y8)[0].any() and not host(y8)[1].any()
    assert np.allclose(f64(rstd), 1e3, rtol=2.0**-20)
    # eps zero: the row's size is of no account as long as its squares are float32 numbers
    x = hidden(4, 700, 5, "f32")
    y = api.rms_norm_forward(x, w, torch.empty_like(x), eps=0.0)
    for size in (2.0**60, 2.0**-60):
        assert torch.equal(api.rms_norm_forward(x * size, w, torch.empty_like(x), eps=0.0), y)
    assert api.rms_norm_forward(x, w) is None


def test_rows_that_are_not_finite_stay_alone():
    x = hidden(6, 900, 3, "bf16")
    x[2, 5], x[4, 899] = float("inf"), float("nan")
    y8 = room(6, 900)
    y = api.rms_norm_forward(x, torch.ones(900, device="cuda"), torch.empty_like(x), y8=y8)
    bad = [False, False, True, False, True, False]
    assert y.isnan().any(dim=1).cpu().tolist() == bad
    assert (host(y8)[1] == 255).any(axis=1).tolist() == bad


def test_no_rows():
    x, w, none = torch.empty(0, 300, device="cuda"), torch.ones(300, device="cuda"), torch.empty(0, device="cuda")
    dw = torch.full_like(w, 3)
    api.rms_norm_forward(x, w, torch.empty_like(x))
    api.rms_norm_backward(x, x, w, none, torch.empty_like(x))
    api.rms_norm_backward(x, x, w, none, torch.empty_like(x), dw)
    assert not dw.any()


def test_results_repeat_to_the_bit():
    first = run(5000, 768, "bf16", residual=True, checkpoint=True)
    second = run(5000, 768, "bf16", residual=True, checkpoint=True)
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_gradient_against_differences():
    # central differences of the float32 forward, h = 2^-6: the third derivative's share is h^2 / 6 of terms of the
    # gradient's own size, the rounding of y 2^-24 / h
    rows, n = 64, 384
    x, dy, d = (hidden(rows, n, s, "f32") for s in (1, 2, 3))
    g = torch.Generator(device="cuda").manual_seed(9)
    w, e = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
    rstd = torch.empty(rows, device="cuda")
    api.rms_norm_forward(x, w, torch.empty_like(x), rstd=rstd, eps=EPS)
    dx, dw = api.rms_norm_backward(dy, x, w, rstd, torch.empty_like(x), torch.empty_like(w))
    h = 2.0**-6
    for grad, by, step in ((dx, d, (d, None)), (dw, e, (None, e))):
        loss = []
        for sign in (h, -h):
            args = [t if s is None else t + sign * s for t, s in zip((x, w), step)]
            y = api.rms_norm_forward(args[0], args[1], torch.empty_like(x), eps=EPS)
            loss.append(float((y.double() * dy.double()).sum()))
        slope = float((grad.double() * by.double()).sum())
        scale = float(grad.double().norm() * by.double().norm())
        assert abs((loss[0] - loss[1]) / (2 * h) - slope) < 1e-3 * scale


def test_refusals():
    x, w = hidden(40, 500, 5, "bf16"), torch.ones(500, device="cuda")
    y, rstd = torch.empty_like(x), torch.ones(40, device="cuda")
    y8 = room(40, 500)
    go = lambda **k: api.rms_norm_forward(k.pop("x", x), k.pop("w", w), k.pop("y", y), **k)  # noqa: E731
    go(y8=y8)
    for bad, err in ((dict(w=w.bfloat16()), TypeError), (dict(w=w[:499]), ValueError), (dict(y=y[:39]), ValueError),
                     (dict(residual=x.float()), TypeError), (dict(rstd=rstd[:39]), ValueError), (dict(x=x.double()), TypeError),
                     (dict(y8=(y8[0].view(torch.uint8), y8[1])), TypeError), (dict(y8=(y8[0], None)), ValueError),
                     (dict(y8=(y8[0], y8[1][:, :3])), ValueError), (dict(y8=room(40, 500, tiles=True)), api.RdfftError),
                     (dict(summed=y), api.RdfftError), (dict(y=x.t()), ValueError), (dict(eps=-1.0), api.RdfftError)):
        with pytest.raises(err):
            go(**bad)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    back = lambda **k: api.rms_norm_backward(*[k.pop(n, v) for n, v in (("dy", y), ("u", x), ("w", w), ("rstd", rstd),  # noqa: E731
                                                                         ("dx", dx), ("dw", dw))], **k)
    back()
    for bad, err in ((dict(u=x.float()), TypeError), (dict(u=(x, x)), TypeError), (dict(dx=x), api.RdfftError),
                     (dict(dw=w), api.RdfftError), (dict(add=x[:, :499]), ValueError), (dict(rstd=rstd.cpu()), ValueError)):
        with pytest.raises(err):
            back(**bad)
    many = hidden(3000, 500, 5, "bf16")
    with pytest.raises(ValueError, match="workspace"):
        api.rms_norm_backward(many, many, w, torch.ones(3000, device="cuda"), torch.empty_like(many), dw,
                              workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_on_another_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(40, 1000, "bf16", residual=True, checkpoint=True, add=True)
    s.synchronize()
