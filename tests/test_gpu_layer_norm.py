"""Layer norm forward and backward against the formulas in 64 bits (the comparison rule of _helpers)."""

import numpy as np
import pytest
import torch

from paper_2511_01385_amd import api
from tests._helpers import assert_close

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def f64(t):
    return t.detach().double().cpu().numpy()


def hidden(rows, n, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda") + 0.3 * torch.randn(n, generator=g, device="cuda")
    return x.to(TYPES[dtype])


def statistics(u):
    mean = u.mean(axis=1, keepdims=True)
    return mean, 1 / np.sqrt(((u - mean) ** 2).mean(axis=1, keepdims=True) + EPS)


def gradients(u, mean, rstd, w, dy):
    xh = (u - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def run(rows, n, dtype, residual=False, checkpoint=False, bias=True, pad=0, seed=0):
    """Forward and backward through the library, each result checked."""
    x = hidden(rows, n + pad, seed, dtype)[:, :n]
    r = hidden(rows, n + 2 * pad, seed + 1, dtype)[:, pad : pad + n] if residual else None
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    w = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
    b = 0.1 * torch.randn(n, generator=g, device="cuda") if bias else None
    dy = torch.randn(rows, n + pad, generator=g, device="cuda").to(TYPES[dtype])[:, :n]
    y = torch.full((rows, n + pad), 5.0, dtype=TYPES[dtype], device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    held = api.checkpoint_like(x) if checkpoint else None
    api.layer_norm_forward(x, w, b, y[:, :n], residual=r, mean=mean, rstd=rstd, checkpoint=held, eps=EPS)
    assert (y[:, n:] == 5).all()

    u = f64(x) + (f64(r) if residual else 0)
    m64, r64 = statistics(u)
    what = f"{dtype} {rows}x{n}"
    assert_close(f64(y[:, :n]), (u - m64) * r64 * f64(w) + (f64(b) if bias else 0), dtype, what + " y")
    # a sum of n float32 terms in a tree is within 2^-20 of the sum of their sizes
    assert np.all(np.abs(f64(mean) - m64[:, 0]) <= 2.0**-20 * np.abs(u).mean(axis=1) + 1e-30)
    assert np.all(np.abs(f64(rstd) / r64[:, 0] - 1) <= 2.0**-18)

    dx = torch.full((rows, n + pad), 5.0, dtype=TYPES[dtype], device="cuda")
    dw, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    if checkpoint:
        # the checkpoint of the norm's input, as the format's own call leaves it for the float32 sum
        total = x.float() + r.float() if residual else x.float()
        codes, scales = api.checkpoint_like(total)
        api.act8_quantize(total, codes, scales)
        assert torch.equal(codes, held[0]) and torch.equal(scales, held[1])
        u = f64(api.act8_dequantize(codes, scales, torch.empty_like(total)))
        api.layer_norm_backward(dy, held, w, mean, rstd, dx[:, :n], dw, db)
    else:
        api.layer_norm_backward(dy, x, w, mean, rstd, dx[:, :n], dw, db, residual=r)
    assert (dx[:, n:] == 5).all()
    # the formula at the statistics that the backward is given
    want = gradients(u, f64(mean)[:, None], f64(rstd)[:, None], f64(w), f64(dy))
    if n > 2:
        assert_close(f64(dx[:, :n]), want[0], dtype, what + " dx")
    else:
        # what is left of g without its parts along 1 and xh is nothing but eps's share and rounding, of terms of g's size
        size = f64(rstd)[:, None] * np.abs(f64(dy) * f64(w)).max(axis=1, keepdims=True)
        assert np.all(np.abs(f64(dx[:, :n]) - want[0]) <= 2.0**-18 * size + 2.0**-8 * np.abs(want[0]))
    assert_close(f64(dw), want[1], "f32", what + " dweight")
    assert_close(f64(db), want[2], "f32", what + " dbias")
    return dx, dw, db


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 2), (3, 7), (5, 8), (1, 33), (17, 256), (4, 511), (130, 513), (33, 768), (300, 769),
                                    (9, 1024), (2, 1025), (40, 2048), (7, 2049), (1, 4096), (300, 4096), (11, 4097),
                                    (5, 8192), (3, 8200), (2, 16383), (300, 16384)])
def test_widths(dtype, rows, n):
    run(rows, n, dtype, seed=n)
    run(rows, n, dtype, residual=True, checkpoint=True, seed=n + 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual,checkpoint,bias,pad", [(True, False, True, 0), (False, True, False, 0),
                                                          (False, False, False, 3), (True, True, True, 5),
                                                          (True, False, True, 8)])
def test_forms(dtype, residual, checkpoint, bias, pad):
    for n in (260, 1027, 4099):
        run(77, n, dtype, residual, checkpoint, bias, pad, seed=n)


@pytest.mark.parametrize("checkpoint", [False, True])
def test_many_rows(checkpoint):
    run(20000, 768, "bf16", residual=True, checkpoint=checkpoint)
    run(9001, 64, "f32", checkpoint=checkpoint)


def test_in_place():
    x, r = hidden(50, 1000, 1, "bf16"), hidden(50, 1000, 2, "bf16")
    w, b = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    want = api.layer_norm_forward(x, w, b, torch.empty_like(x), residual=r)
    for target in (0, 1):
        pair = [x.clone(), r.clone()]
        api.layer_norm_forward(pair[0], w, b, pair[target], residual=pair[1])
        assert torch.equal(pair[target], want) and torch.equal(pair[1 - target], (r, x)[target])
    mean, rstd = torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    api.layer_norm_forward(x, w, b, torch.empty_like(x), mean=mean, rstd=rstd)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    dx = api.layer_norm_backward(r, x, w, mean, rstd, torch.empty_like(x), dw, db)[0]
    dy = r.clone()
    api.layer_norm_backward(dy, x, w, mean, rstd, dy, dw, db)
    assert torch.equal(dy, dx)


def test_slices_side_by_side_and_refusals():
    both = hidden(40, 1000, 4, "bf16")
    dy, dx = both[:, :500], both[:, 500:]
    x, w = hidden(40, 500, 5, "bf16"), torch.ones(500, device="cuda")
    mean, rstd = torch.zeros(40, device="cuda"), torch.ones(40, device="cuda")
    want = api.layer_norm_backward(dy.clone(), x, w, mean, rstd, torch.empty_like(x), torch.empty_like(w), torch.empty_like(w))[0]
    dw, db = torch.empty_like(w), torch.empty_like(w)
    assert torch.equal(api.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)[0], want)
    back = lambda **k: api.layer_norm_backward(*[k.get(n, v) for n, v in (  # noqa: E731
        ("dy", dy), ("x", x), ("w", w), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db))])
    for bad, err in ((dict(x=x.float()), TypeError), (dict(w=w.bfloat16()), TypeError), (dict(w=w[:499]), ValueError),
                     (dict(dx=dx[:39]), ValueError), (dict(mean=mean[:39]), ValueError), (dict(dw=w.cpu()), ValueError),
                     (dict(dx=torch.empty(500, 40, dtype=x.dtype, device="cuda").t()), ValueError),
                     (dict(dx=x), api.RdfftError), (dict(x=(x, x)), TypeError), (dict(dy=dy.double()), TypeError)):
        with pytest.raises(err):
            back(**bad)
    with pytest.raises(ValueError):
        api.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_constant_rows_and_large_means():
    # variance zero: y is the bias; a mean a thousand times the deviation loses only what float32 inputs have lost
    x = torch.full((3, 700), 2.5, device="cuda")
    w, b = torch.ones(700, device="cuda"), torch.linspace(-1, 1, 700, device="cuda")
    y = api.layer_norm_forward(x, w, b, torch.empty_like(x))
    assert torch.equal(y, b.expand(3, -1))
    x = torch.randn(5, 700, device="cuda") + 1000
    u = f64(x)
    m, r = statistics(u)
    y = api.layer_norm_forward(x, w, b, torch.empty_like(x))
    # the mean is off by half an ulp of 1000 (2^-15) at the least, next to a deviation of one
    assert np.abs(f64(y) - ((u - m) * r + f64(b))).max() < 4 * 2.0**-14


def test_rows_that_are_not_finite_stay_alone():
    x = hidden(6, 900, 3, "bf16")
    x[2, 5], x[4, 899] = float("inf"), float("nan")
    w, b = torch.ones(900, device="cuda"), torch.zeros(900, device="cuda")
    y = api.layer_norm_forward(x, w, b, torch.empty_like(x))
    bad = y.isnan().any(dim=1).cpu()
    assert bad.tolist() == [False, False, True, False, True, False]


def test_no_rows():
    x = torch.empty(0, 300, device="cuda")
    w = torch.ones(300, device="cuda")
    dw, db = torch.full_like(w, 3), torch.full_like(w, 3)
    none = torch.empty(0, device="cuda")
    api.layer_norm_forward(x, w, w, torch.empty_like(x))
    api.layer_norm_backward(x, x, w, none, none, torch.empty_like(x), dw, db)
    assert not dw.any() and not db.any()


def test_results_repeat_to_the_bit():
    first = run(5000, 768, "bf16", residual=True, checkpoint=True)
    second = run(5000, 768, "bf16", residual=True, checkpoint=True)
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_gradient_against_differences():
    # d/dt of sum(y dy) at x + t d, w + t e, b + t f by central differences of the float32 forward, h = 2^-6:
    # the third derivative's share is h^2 / 6 of terms of the gradient's own size, the rounding of y 2^-24 / h
    rows, n = 64, 384
    x, dy, d = (hidden(rows, n, s, "f32") for s in (1, 2, 3))
    g = torch.Generator(device="cuda").manual_seed(9)
    w, b, e, f = (torch.randn(n, generator=g, device="cuda") for _ in range(4))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    api.layer_norm_forward(x, w, b, torch.empty_like(x), mean=mean, rstd=rstd, eps=EPS)
    dx, dw, db = api.layer_norm_backward(dy, x, w, mean, rstd, torch.empty_like(x), torch.empty_like(w), torch.empty_like(w))
    h = 2.0**-6
    for grad, step in (((dx, d),), (d, None, None)), (((dw, e),), (None, e, None)), (((db, f),), (None, None, f)):
        loss = []
        for sign in (h, -h):
            args = [t if s is None else t + sign * s for t, s in zip((x, w, b), step)]
            y = api.layer_norm_forward(args[0], args[1], args[2], torch.empty_like(x), eps=EPS)
            loss.append(float((y.double() * dy.double()).sum()))
        (gr, di), = grad
        slope = float((gr.double() * di.double()).sum())
        scale = float(gr.double().norm() * di.double().norm())
        assert abs((loss[0] - loss[1]) / (2 * h) - slope) < 1e-3 * scale


def test_on_another_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(40, 1000, "bf16", residual=True, checkpoint=True)
    s.synchronize()
