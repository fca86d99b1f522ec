"""What RMS norm and the operators in 8-bit floating point refuse, on the host before any HIP call (no GPU needed): every
call below must fail validation or have nothing to do, so nothing is ever launched from here."""

import math

import pytest
import torch

from paper_2511_01385_amd import _lib, api

EINVAL, EUNSUP, OK = _lib.RDFFT_EINVAL, _lib.RDFFT_EUNSUPPORTED, _lib.RDFFT_OK
F32, BF16, F16 = _lib.RDFFT_F32, _lib.RDFFT_BF16, _lib.RDFFT_F16

# fake addresses, never dereferenced, 1 GiB apart
P = [0x7F0000000000 + (i << 30) for i in range(20)]


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def call(lib, name, fields, *args):
    order = _lib._FIELDS[name].split()
    assert set(fields) <= set(order)
    return getattr(lib, name)(_lib.pack[name](*[fields.get(f, 0) for f in order]), *args)


def pack(codes, ld, scales, lds, block_rows):
    return None if codes is None else _lib.pack["fp8"](codes, ld, scales, lds, block_rows)


def quantize(lib, x=P[0], ldx=200, codes=P[1], ld=208, scales=P[2], lds=4, block_rows=1, c_codes=P[3], c_ld=304, c_scales=P[4],
             c_lds=4, c_block_rows=1, rows=300, n=200, dtype=BF16):
    return lib.fp8_quantize(x, ldx, pack(codes, ld, scales, lds, block_rows), pack(c_codes, c_ld, c_scales, c_lds, c_block_rows),
                            rows, n, dtype, None)


@pytest.mark.parametrize("change,want", [
    (dict(x=0), EINVAL), (dict(x=P[0] + 1), EINVAL), (dict(ldx=199), EINVAL), (dict(rows=-1), EINVAL), (dict(n=0), EINVAL),
    (dict(dtype=3), EINVAL), (dict(codes=None, c_codes=None), EINVAL), (dict(codes=0), EINVAL), (dict(scales=0), EINVAL),
    (dict(c_codes=0), EINVAL), (dict(c_scales=0), EINVAL), (dict(codes=P[1] + 8), EINVAL), (dict(scales=P[2] + 2), EINVAL),
    (dict(c_codes=P[3] + 4), EINVAL), (dict(ld=200), EINVAL), (dict(ld=192), EINVAL), (dict(lds=2), EINVAL), (dict(lds=1), EINVAL),
    (dict(c_ld=300), EINVAL), (dict(c_ld=296), EINVAL), (dict(c_lds=3), EINVAL), (dict(c_lds=2), EINVAL),
    (dict(block_rows=0), EINVAL), (dict(block_rows=32), EINVAL), (dict(c_block_rows=2), EINVAL),
    (dict(block_rows=128), EINVAL),  # and columns by rows
    (dict(codes=P[0] + 16), EINVAL), (dict(c_scales=P[1] + 64), EINVAL), (dict(scales=P[3] + 32), EINVAL),
    (dict(c_codes=P[1]), EINVAL), (dict(rows=1 << 62), EINVAL), (dict(rows=0, x=0, codes=None, c_codes=None), OK),
    (dict(rows=1, n=(1 << 29) + 16, ldx=(1 << 29) + 16, codes=P[2], ld=(1 << 29) + 16, scales=P[8], lds=1 << 23, c_codes=None), EUNSUP),
])
def test_quantize(lib, change, want):
    assert quantize(lib, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(codes=0), EINVAL), (dict(scales=0), EINVAL), (dict(out=0), EINVAL), (dict(out=P[0] + 1), EINVAL), (dict(ldo=199), EINVAL),
    (dict(ld=207), EINVAL), (dict(lds=3), EINVAL), (dict(codes=P[1] + 1), EINVAL), (dict(block_rows=64), EINVAL),
    (dict(out=P[1] + 64), EINVAL), (dict(out=P[2]), EINVAL), (dict(n=-1), EINVAL), (dict(dtype=-1), EINVAL),
    (dict(rows=0, codes=0, scales=0, out=0), OK),
])
def test_dequantize(lib, change, want):
    a = {**dict(codes=P[1], ld=208, scales=P[2], lds=4, block_rows=1, out=P[0], ldo=200, rows=300, n=200, dtype=BF16), **change}
    assert lib.fp8_dequantize(pack(a["codes"], a["ld"], a["scales"], a["lds"], a["block_rows"]), a["out"], a["ldo"], a["rows"],
                              a["n"], a["dtype"], None) == want


def test_dequantize_from_nothing(lib):
    assert lib.fp8_dequantize(None, P[0], 200, 300, 200, BF16, None) == EINVAL


NORM = dict(x=P[0], ldx=64, residual=P[1], ldr=64, weight=P[2], y=P[3], ldy=64, summed=P[4], lds=64, rstd=P[5], codes=P[6],
            scales=P[7], codes8=P[8], ld8=64, scales8=P[9], lds8=4, block_rows8=1)


@pytest.mark.parametrize("change,want", [
    (dict(x=0), EINVAL), (dict(weight=0), EINVAL), (dict(ldx=63), EINVAL), (dict(ldr=60), EINVAL), (dict(ldy=1), EINVAL),
    (dict(lds=63), EINVAL), (dict(x=P[0] + 1), EINVAL), (dict(weight=P[2] + 2), EINVAL), (dict(rstd=P[5] + 1), EINVAL),
    (dict(codes=0), EINVAL), (dict(scales=0), EINVAL), (dict(codes8=0), EINVAL), (dict(scales8=0), EINVAL),
    (dict(codes8=P[8] + 8), EINVAL), (dict(ld8=72), EINVAL), (dict(lds8=1), EINVAL), (dict(scales8=P[9] + 1), EINVAL),
    (dict(block_rows8=128), EINVAL), (dict(block_rows8=0), EINVAL),
    (dict(y=P[0] + 2), EINVAL), (dict(y=P[0], ldy=128), EINVAL), (dict(summed=P[1] + 2), EINVAL),
    (dict(summed=P[3]), EINVAL), (dict(y=P[0], summed=P[0]), EINVAL),  # each other
    (dict(residual=P[3] + 64), EINVAL), (dict(rstd=P[0] + 64), EINVAL), (dict(codes8=P[0]), EINVAL), (dict(codes8=P[3]), EINVAL),
    (dict(scales8=P[8] + 64), EINVAL), (dict(y=P[2]), EINVAL), (dict(codes=P[4] + 8), EINVAL), (dict(codes=P[1]), EINVAL),
])
def test_rms_norm_forward(lib, change, want):
    assert call(lib, "rms_norm_forward", {**NORM, **change}, 4, 64, 1e-6, BF16, None) == want


def test_rms_norm_forward_sizes(lib):
    go = lambda rows=4, n=64, eps=1e-6, dtype=BF16: call(lib, "rms_norm_forward", NORM, rows, n, eps, dtype, None)  # noqa: E731
    assert go(rows=0) == OK and go(rows=-1) == EINVAL and go(n=0) == EINVAL and go(dtype=7) == EINVAL and go(n=16385) == EUNSUP
    assert go(eps=-1e-9) == EINVAL and go(eps=math.nan) == EINVAL and go(eps=math.inf) == EINVAL
    assert lib.rms_norm_forward(None, 4, 64, 1e-6, BF16, None) == EINVAL


GRAD = dict(dy=P[0], ldg=64, u=P[1], ldu=64, weight=P[2], rstd=P[3], add=P[4], lda=64, dx=P[5], ldd=64, dweight=P[6],
            workspace=P[7], workspace_bytes=1 << 20)


@pytest.mark.parametrize("change,want", [
    (dict(dy=0), EINVAL), (dict(weight=0), EINVAL), (dict(rstd=0), EINVAL), (dict(dx=0), EINVAL), (dict(u=0), EINVAL),
    (dict(u=0, codes=P[8]), EINVAL), (dict(ldg=10), EINVAL), (dict(ldu=63), EINVAL), (dict(lda=1), EINVAL), (dict(ldd=63), EINVAL),
    (dict(workspace=0), EINVAL), (dict(workspace_bytes=16), EINVAL), (dict(workspace=P[7] + 8), EINVAL),
    (dict(dx=P[0] + 2), EINVAL), (dict(dx=P[0], ldd=72), EINVAL), (dict(dx=P[1]), EINVAL), (dict(dx=P[4] + 128), EINVAL),
    (dict(dweight=P[0] + 4), EINVAL), (dict(dweight=P[2]), EINVAL), (dict(workspace=P[5]), EINVAL), (dict(workspace=P[4] + 16), EINVAL),
    (dict(rstd=P[3] + 2), EINVAL), (dict(dweight=P[6] + 1), EINVAL),
])
def test_rms_norm_backward(lib, change, want):
    assert call(lib, "rms_norm_backward", {**GRAD, **change}, 4000, 64, BF16, None) == want


def test_rms_norm_backward_sizes(lib):
    go = lambda rows=4, n=64, dtype=BF16, **k: call(lib, "rms_norm_backward", {**GRAD, **k}, rows, n, dtype, None)  # noqa: E731
    assert go(rows=-1) == EINVAL and go(n=0) == EINVAL and go(dtype=9) == EINVAL and go(n=16385) == EUNSUP
    assert go(rows=0, dweight=0) == OK
    assert lib.rms_norm_backward(None, 4, 64, BF16, None) == EINVAL
    need = lib.rms_norm_backward_workspace
    assert need(-1, 64) == EINVAL and need(4, 0) == EINVAL and need(4, 16385) == EUNSUP
    assert need(1, 64) == 0 < need(100000, 64) and need(1 << 40, 16384) <= 64 << 20


LINEAR = dict(x=P[0], ldx=64, x_scales=P[1], ldxs=4, x_block_rows=1, w=P[2], ldw=64, w_scales=P[3], ldws=4, w_block_rows=128,
              bias=P[4], y=P[5], ldy=96, codes=P[6], scales=P[7], workspace=P[8], workspace_bytes=1 << 29)


@pytest.mark.parametrize("change,want", [
    (dict(x=0), EINVAL), (dict(w=0), EINVAL), (dict(y=0), EINVAL), (dict(x_scales=0), EINVAL), (dict(w_scales=0), EINVAL),
    (dict(x=P[0] + 8), EINVAL), (dict(w=P[2] + 1), EINVAL), (dict(x_scales=P[1] + 2), EINVAL), (dict(ldx=72), EINVAL),
    (dict(ldx=48), EINVAL), (dict(ldw=63), EINVAL), (dict(ldxs=2), EINVAL), (dict(ldxs=0), EINVAL), (dict(x_block_rows=0), EINVAL),
    (dict(w_block_rows=127), EINVAL), (dict(w_block_rows=1, ldws=3), EINVAL), (dict(ldy=95), EINVAL), (dict(y=P[5] + 1), EINVAL),
    (dict(bias=P[4] + 1), EINVAL), (dict(codes=0), EINVAL), (dict(scales=0), EINVAL), (dict(residual=P[9], ldr=80), EINVAL),
    (dict(y=P[0]), EINVAL), (dict(y=P[3]), EINVAL), (dict(y=P[4] + 32), EINVAL), (dict(residual=P[5] + 2, ldr=96), EINVAL),
    (dict(residual=P[5], ldr=100), EINVAL), (dict(codes=P[5]), EINVAL), (dict(ldx=(1 << 21) + 16), EUNSUP),
    (dict(ldw=(1 << 21) + 16), EUNSUP), (dict(workspace=0), EINVAL), (dict(workspace_bytes=256), EINVAL),
    (dict(workspace=P[8] + 4), EINVAL), (dict(workspace=P[5]), EINVAL),
])
def test_linear_forward(lib, change, want):
    tokens, d_in, d_out = 96, 64, 96
    if any(k.startswith("workspace") for k in change):  # a size whose k is split
        tokens, d_in = 96, 65536
        change = {"ldx": d_in, "ldw": d_in, "ldxs": 512, "ldws": 512, **change}
        assert lib.linear_fp8_forward_workspace(d_in, d_out, tokens, BF16) > 256
    assert call(lib, "linear_fp8_forward", {**LINEAR, **change}, d_in, d_out, tokens, 0, BF16, None) == want


def test_linear_forward_sizes(lib):
    go = lambda d_in=64, d_out=96, tokens=96, act=0, dtype=BF16: call(  # noqa: E731
        lib, "linear_fp8_forward", LINEAR, d_in, d_out, tokens, act, dtype, None)
    assert go(tokens=0) == OK and go(tokens=-1) == EINVAL and go(d_in=0) == EINVAL and go(d_out=0) == EINVAL
    assert go(act=4) == EINVAL and go(act=-1) == EINVAL and go(dtype=3) == EINVAL
    assert go(d_in=(1 << 20) + 1) == EUNSUP and go(tokens=(1 << 22) + 1) == EUNSUP
    assert lib.linear_fp8_forward(None, 64, 96, 4, 0, BF16, None) == EINVAL
    need = lib.linear_fp8_forward_workspace
    assert need(64, 0, 4, BF16) == EINVAL and need(1 << 21, 64, 4, BF16) == EUNSUP and need(4096, 4096, 64, BF16) == 0


BACK = dict(dy=P[0], ldg=96, x=P[1], ldx=304, x_scales=P[2], ldxs=4, x_block_rows=1, w=P[3], ldw=96, w_scales=P[4], ldws=4,
            w_block_rows=128, add=P[5], lda=64, dx=P[6], ldd=64, dw=P[7], lddw=64, db=P[8], workspace=P[9], workspace_bytes=1 << 29)


@pytest.mark.parametrize("change,want", [
    (dict(dy=0), EINVAL), (dict(x=0), EINVAL), (dict(w=0), EINVAL), (dict(x_scales=0), EINVAL), (dict(w_scales=0), EINVAL),
    (dict(ldg=95), EINVAL), (dict(ldx=300), EINVAL), (dict(ldx=288), EINVAL), (dict(ldw=80), EINVAL), (dict(ldxs=2), EINVAL),
    (dict(x=P[1] + 4), EINVAL), (dict(w_scales=P[4] + 1), EINVAL), (dict(x_block_rows=3), EINVAL), (dict(lda=63), EINVAL),
    (dict(ldd=63), EINVAL), (dict(lddw=60), EINVAL), (dict(dw=P[7] + 1), EINVAL), (dict(dx=P[0]), EINVAL), (dict(dx=P[5], ldd=72), EINVAL),
    (dict(dw=P[1] + 64), EINVAL), (dict(db=P[3]), EINVAL), (dict(db=P[7] + 64), EINVAL), (dict(dw=P[5]), EINVAL),
    (dict(workspace=0), EINVAL), (dict(workspace_bytes=1000), EINVAL), (dict(workspace=P[9] + 8), EINVAL),
    (dict(workspace=P[2]), EINVAL), (dict(workspace=P[6]), EINVAL), (dict(ldw=(1 << 21) + 16), EUNSUP),
    (dict(dx=0, dw=0, db=0), OK),
])
def test_linear_backward(lib, change, want):
    assert call(lib, "linear_fp8_backward", {**BACK, **change}, 64, 96, 300, 0, BF16, None) == want


def test_linear_backward_sizes(lib):
    go = lambda d_in=64, d_out=96, tokens=300, act=0, dtype=BF16, **k: call(  # noqa: E731
        lib, "linear_fp8_backward", {**BACK, **k}, d_in, d_out, tokens, act, dtype, None)
    assert go(tokens=-1) == EINVAL and go(act=7) == EINVAL and go(dtype=5) == EINVAL and go(d_in=(1 << 20) + 1) == EUNSUP
    assert go(act=2) == EINVAL  # no checkpoint
    assert lib.linear_fp8_backward(None, 64, 96, 4, 0, BF16, None) == EINVAL
    need = lib.linear_fp8_backward_workspace
    assert need(64, 0, 4, 1, 1, 1, BF16) == EINVAL
    # dz by rows and by columns, in rows of 16 codes and of 4 scales, and the sums of 128 tokens each
    assert need(64, 96, 300, 0, 0, 1, BF16) >= 3 * 96 * 4
    assert need(64, 96, 300, 1, 0, 0, BF16) >= 300 * (96 + 4) and need(64, 96, 300, 0, 1, 0, BF16) >= 96 * (304 + 4)


def test_python_refuses():
    cpu = torch.empty(4, 128)
    held = api.fp8_like(cpu)
    for go in (lambda: api.fp8_quantize(cpu, held), lambda: api.fp8_quantize(cpu), lambda: api.fp8_dequantize(held, cpu),
               lambda: api.rms_norm_forward(cpu, torch.ones(128), cpu), lambda: api.linear_fp8_forward(held, held, cpu),
               lambda: api.linear_fp8_backward(cpu, held, held, dx=cpu), lambda: api.rms_norm_backward(cpu, cpu, cpu, cpu, cpu),
               lambda: api.linear_fp8_forward(held, held, cpu, activation="tanh")):
        with pytest.raises(ValueError):
            go()


@pytest.mark.parametrize("rows,n", [(1, 1), (3, 200), (300, 129), (0, 64)])
def test_fp8_like(rows, n):
    x = torch.empty(rows, n)
    for columns in (False, True):
        r, c = (n, rows) if columns else (rows, n)
        for tiles in (False, True):
            codes, scales = api.fp8_like(x, columns=columns, tiles=tiles)
            assert codes.shape == (r, c) and codes.dtype is torch.float8_e4m3fn and scales.dtype is torch.uint8
            assert scales.shape == (-(-r // 128) if tiles else r, -(-c // 128))
            assert r < 2 or c == 0 or (codes.stride(0) % 16 == 0 and scales.stride(0) % 4 == 0)
