"""RMS norm and the operators in 8-bit floating point through the native module: it takes plain calls and slices itself (the
long way is closed here), hands back what is not plainly right, and gives the long way's results to the bit."""

import pytest
import torch

from paper_2511_01385_amd import _lib, api
from tests._fp8 import room

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


class HandsBack:
    def __getattr__(self, name):
        return lambda *args: None


def made(rows, n, dtype, seed, wider=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, n + wider), generator=g, device="cuda").to(dtype)[:, :n]


def run_all(dtype, wider, rows=137, n=200, d_out=80):
    """Every operator, every argument, from inputs that depend on the sizes alone."""
    x, r, dy = (made(rows, n, dtype, i, wider) for i in (1, 2, 3))
    weight = made(1, n, torch.float32, 4)[0]
    out = []
    pad = wider % 3
    for tiles in (False, True):
        held, columns = room(rows, n, tiles, pad), room(n, rows, tiles, pad)
        api.fp8_quantize(x, held, columns=columns)
        out += [*held, *columns, api.fp8_dequantize(held, made(rows, n, dtype, 6, wider))]
    rstd, ck, y8 = torch.empty(rows, device="cuda"), api.checkpoint_like(x), room(rows, n, pad=pad)
    u, y = made(rows, n, dtype, 7, wider), made(rows, n, dtype, 8, wider)
    api.rms_norm_forward(x, weight, y, residual=r, summed=u, rstd=rstd, checkpoint=ck, y8=y8)
    out += [u, y, rstd, *ck, *y8]
    for source in (u, ck):
        out += api.rms_norm_backward(dy, source, weight, rstd, made(rows, n, dtype, 6, wider), torch.empty_like(weight), add=r)
    w = made(d_out, n, torch.float32, 9)
    w8, w8t, x8t = room(d_out, n, True, pad), room(n, d_out, True, pad), room(n, rows, pad=pad)
    api.fp8_quantize(w, w8, columns=w8t), api.fp8_quantize(y, columns=x8t)
    b, res, dout = made(1, d_out, dtype, 10)[0], made(rows, d_out, dtype, 11, wider), made(rows, d_out, dtype, 12, wider)
    z8 = api.checkpoint_like(res)
    out += [api.linear_fp8_forward(y8, w8, made(rows, d_out, dtype, 6, wider), bias=b, activation="gelu", residual=res,
                                   checkpoint=z8), *z8]
    out += api.linear_fp8_backward(dout, x8t, w8t, dx=made(rows, n, dtype, 6, wider), dw=made(d_out, n, dtype, 6, wider),
                                   db=torch.empty_like(b), activation="gelu", checkpoint=z8, add=r)
    return [(t.view(torch.uint8) if t.dtype is torch.float8_e4m3fn else t).clone() for t in out]


@pytest.mark.parametrize("wider", [0, 8, 3])
@pytest.mark.parametrize("dtype", DTYPES)
def test_taken_and_the_same(dtype, wider, monkeypatch):
    def closed(*args):
        raise AssertionError("the long way was taken")

    with monkeypatch.context() as m:
        m.setattr(api, "_first", closed)
        got = run_all(dtype, wider)
    with monkeypatch.context() as m:
        m.setattr(_lib, "_binding", HandsBack())
        want = run_all(dtype, wider)
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and torch.equal(a, b)


def test_hands_back():
    module, device = _lib.binding(), torch.cuda.current_device()
    stream = torch.cuda.current_stream().cuda_stream
    x = made(4, 64, torch.bfloat16, 1)
    codes, scales = room(4, 64)

    def quantize(x=x, codes=codes, scales=scales, c=None, s=None, device=device, stream=stream):
        return module.fp8_quantize(x, codes, scales, c, s, device, stream)

    assert quantize() == 0
    for bad in (dict(x=None), dict(x=3), dict(x=x.cpu()), dict(x=x.double()), dict(x=x[0]), dict(x=x[:3]), dict(x=x.t()),
                dict(codes=codes[:, :63]), dict(codes=codes.view(torch.uint8)), dict(codes=None), dict(scales=None),
                dict(scales=scales.view(torch.int8)), dict(scales=scales[:3]), dict(scales=scales.cpu()), dict(c=codes),
                dict(device=device + 1), dict(stream=None)):
        assert quantize(**bad) is None, bad
    assert module.fp8_quantize(x, codes, scales) is None


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    if not native:
        monkeypatch.setattr(_lib, "_binding", HandsBack())
    x, w = room(40, 300, junk=False), room(200, 300, True, junk=False)
    y = torch.empty(40, 200, dtype=torch.bfloat16, device="cuda")
    go = lambda **k: api.linear_fp8_forward(k.pop("x", x), k.pop("w", w), k.pop("y", y), **k)  # noqa: E731
    go()
    odd = torch.empty(40, 301, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :300]
    for bad, err in ((dict(x=(x[0], None)), ValueError), (dict(x=(x[0], x[1][:, :2])), ValueError),
                     (dict(x=(x[0][:, :299], x[1])), ValueError), (dict(w=(w[0].view(torch.uint8), w[1])), TypeError),
                     (dict(x=(odd, x[1])), api.RdfftError), (dict(y=y.double()), TypeError), (dict(y=y[:39]), ValueError),
                     (dict(bias=torch.empty(200, device="cuda")), TypeError), (dict(residual=y[:, :199]), ValueError),
                     (dict(activation="tanh"), ValueError), (dict(checkpoint=(y, y)), TypeError), (dict(w=(w[0], w[1].cpu())), ValueError)):
        with pytest.raises(err):
            go(**bad)
    dy, wt, xt = y, room(300, 200, True, junk=False), room(300, 40, junk=False)
    dx, dw = torch.empty(40, 300, dtype=y.dtype, device="cuda"), torch.empty(200, 300, dtype=y.dtype, device="cuda")
    back = lambda **k: api.linear_fp8_backward(dy, k.pop("x", xt), k.pop("w", wt), **{**dict(dx=dx, dw=dw), **k})  # noqa: E731
    back()
    for bad, err in ((dict(x=None), ValueError), (dict(w=None), ValueError), (dict(activation="gelu"), ValueError),
                     (dict(x=x), ValueError), (dict(dw=dw[:, :299]), ValueError), (dict(dx=dy), ValueError), (dict(add=y), ValueError),
                     (dict(db=torch.empty(200, device="cuda")), TypeError),
                     (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), ValueError)):
        with pytest.raises(err):
            back(**bad)
    with pytest.raises(ValueError):
        api.fp8_quantize(y)
    with pytest.raises(api.RdfftError):
        api.fp8_quantize(y, room(40, 200, True), columns=room(200, 40))
    with pytest.raises(ValueError):
        api.fp8_dequantize((x[0], x[1], x[1]), dx)


def test_no_memory_for_the_workspace():
    """torch's own error, and the next call with room is fine."""
    tokens, d_out = 8192, 16384
    dy = torch.ones((tokens, d_out), dtype=torch.bfloat16, device="cuda")
    held = api.act8_quantize(dy, *api.checkpoint_like(dy))
    xt = room(16, tokens, junk=False)
    dw = torch.empty((d_out, 16), dtype=torch.bfloat16, device="cuda")

    def call():
        return api.linear_fp8_backward(dy, xt, None, dw=dw, activation="relu", checkpoint=held)

    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (8 << 20)) / total)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            call()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    call()
    assert not dw.any()


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, give what one after the other gives."""
    tokens, d, d_out = 512, 768, 640
    jobs = []
    for seed in (1, 2):
        x, w, dy = made(tokens, d, torch.bfloat16, seed), made(d_out, d, torch.bfloat16, seed + 10), made(tokens, d_out, torch.bfloat16, seed + 20)
        xt, wt = room(d, tokens), room(d, d_out, True)
        api.fp8_quantize(x, columns=xt), api.fp8_quantize(w, columns=wt)
        out = [torch.empty_like(x), torch.empty_like(w), torch.empty(d_out, dtype=x.dtype, device="cuda")]
        jobs.append((dy, xt, wt, out))
    want = [[t.clone() for t in api.linear_fp8_backward(dy, xt, wt, dx=o[0], dw=o[1], db=o[2])] for dy, xt, wt, o in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(5):
        for s, (dy, xt, wt, o) in zip(streams, jobs):
            with torch.cuda.stream(s):
                for t in o:
                    t.zero_()
                api.linear_fp8_backward(dy, xt, wt, dx=o[0], dw=o[1], db=o[2])
        torch.cuda.synchronize()
        for (_, _, _, o), ref in zip(jobs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, ref))
