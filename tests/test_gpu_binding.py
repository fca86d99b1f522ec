"""The native module that the operators around the adapter are called through: it takes plain calls and slices itself
(the long way is closed here), hands back what is not plainly right, and gives the long way's results to the bit."""

import pytest
import torch

from paper_2511_01385_amd import _lib, api

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def made(rows, n, dtype, seed, wider=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, n + wider), generator=g, device="cuda").to(dtype)[:, :n]


def run_all(dtype, wider, rows=37, n=96, d_out=80):
    """Every operator, every argument, from inputs that depend on the sizes alone."""
    x, r, dy = (made(rows, n, dtype, i, wider) for i in (1, 2, 3))
    weight, bias = made(1, n, torch.float32, 4)[0], made(1, n, torch.float32, 5)[0]
    out = []
    held = api.act8_quantize(x, *api.checkpoint_like(x))
    out += [*held, api.act8_dequantize(*held, made(rows, n, dtype, 6, wider))]
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    held = api.checkpoint_like(x)
    out += [api.layer_norm_forward(x, weight, bias, made(rows, n, dtype, 6, wider), residual=r, mean=mean, rstd=rstd,
                                   checkpoint=held), mean, rstd, *held]
    for source, residual in ((x, r), (held, None)):
        out += api.layer_norm_backward(dy, source, weight, mean, rstd, made(rows, n, dtype, 6, wider),
                                       torch.empty_like(weight), torch.empty_like(bias), residual=residual)
    w, b = made(d_out, n, dtype, 7, wider), made(1, d_out, dtype, 8)[0]
    res, dout = made(rows, d_out, dtype, 9, wider), made(rows, d_out, dtype, 10, wider)
    held = api.checkpoint_like(res)
    out += [api.linear_forward(x, w, made(rows, d_out, dtype, 6, wider), bias=b, activation="gelu", residual=res,
                               checkpoint=held), *held]
    out += api.linear_backward(dout, x, w, dx=made(rows, n, dtype, 6, wider), dw=made(d_out, n, dtype, 6, wider),
                               db=torch.empty_like(b), activation="gelu", checkpoint=held, add=r)
    return [t.clone() for t in out]


@pytest.mark.parametrize("wider", [0, 8, 3])
@pytest.mark.parametrize("dtype", DTYPES)
def test_taken_and_the_same(dtype, wider, monkeypatch):
    class HandsBack:
        def __getattr__(self, name):
            return lambda *args: None

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
    codes, scales = api.checkpoint_like(x)

    def quantize(x=x, codes=codes, scales=scales, device=device, stream=stream):
        return module.act8_quantize(x, codes, scales, device, stream)

    assert quantize() == 0
    for bad in (dict(x=None), dict(x=3), dict(x=x.cpu()), dict(x=x.double()), dict(x=x[0]), dict(x=x[:3]), dict(x=x.t()),
                dict(x=x.expand(4, 64)[:, ::2]), dict(codes=codes[:, :63]), dict(codes=scales), dict(codes=None),
                dict(scales=None), dict(scales=scales[:, :1]), dict(scales=scales.cpu()), dict(device=device + 1),
                dict(device="0"), dict(stream=None), dict(stream=1 << 70)):
        assert quantize(**bad) is None, bad
    assert module.act8_quantize(x, codes, scales) is None

    # (the long way takes what only the native one does not)
    weight, y = torch.ones(64, device="cuda"), torch.empty_like(x)
    assert torch.equal(api.layer_norm_forward(x, weight, None, y, eps=0).clone(),
                       api.layer_norm_forward(x, weight, None, y, eps=0.0))


def test_short_workspace():
    x, mean = made(300, 64, torch.float32, 1), torch.zeros(300, device="cuda")
    weight = torch.ones(64, device="cuda")
    need = api.layer_norm_backward_workspace(300, 64)
    assert need > 0
    short = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="workspace"):
        api.layer_norm_backward(x, x, weight, mean, mean, torch.empty_like(x), weight.clone(), weight.clone(), workspace=short)


def test_statuses_reach_the_caller():
    """What only the C entry refuses: here an output over half of the input."""
    buffer = made(1, 4 * 64 + 32, torch.float32, 1)[0]
    x, y = buffer[:256].view(4, 64), buffer[32:].view(4, 64)
    with pytest.raises(api.RdfftError):
        api.layer_norm_forward(x, torch.ones(64, device="cuda"), None, y)


def test_half_a_checkpoint_is_refused():
    x, w, one = made(4, 64, torch.bfloat16, 1), made(64, 64, torch.bfloat16, 2), torch.ones(64, device="cuda")
    mean = torch.zeros(4, device="cuda")
    codes, scales = api.checkpoint_like(x)
    for half in ((None, scales), (codes, None), ()):
        for call in (lambda: api.layer_norm_forward(x, one, None, torch.empty_like(x), checkpoint=half),
                     lambda: api.linear_forward(x, w, torch.empty_like(x), checkpoint=half),
                     lambda: api.linear_backward(x, None, w, dx=torch.empty_like(x), activation="gelu", checkpoint=half),
                     lambda: api.layer_norm_backward(x, half, one, mean, mean, torch.empty_like(x), one.clone(), one.clone())):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("native", [True, False])
def test_no_memory_for_the_workspace(native, monkeypatch):
    """Both ways raise torch's own error, and the next call with room is fine."""
    class HandsBack:
        def __getattr__(self, name):
            return lambda *args: None

    if not native:
        monkeypatch.setattr(_lib, "_binding", HandsBack())
    tokens, d_out = 8192, 16384
    dy = torch.ones((tokens, d_out), dtype=torch.bfloat16, device="cuda")
    held = api.act8_quantize(dy, *api.checkpoint_like(dy))
    db = torch.empty(d_out, dtype=torch.bfloat16, device="cuda")

    def call():
        return api.linear_backward(dy, None, None, db=db, activation="relu", checkpoint=held)

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
    assert (db == tokens).all()
