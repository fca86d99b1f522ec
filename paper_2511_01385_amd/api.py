"""PyTorch-facing binding of the C ABI (same names as include/rdfft.h).

Torch supplies device memory and the current stream; every call passes raw
pointers and sizes to ``librdfft.so`` and checks the returned status.  No torch
operation touches the data.
"""

from __future__ import annotations

import ctypes
import functools

import torch

from . import _lib


class RdfftError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {_lib.status_string(status)}")
        self.status = status


_CODES = {torch.float32: _lib.RDFFT_F32, torch.bfloat16: _lib.RDFFT_BF16, torch.float16: _lib.RDFFT_F16}

# The current device and its current stream as plain integers.  The public calls build a Stream
# object each time (3 us of a call that takes 9 us on the host with a 5 us kernel); they
# serve where this torch has no raw ones.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"rdfft supports float32, bfloat16 and float16 storage, got {t.dtype}")
    return code


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(t: torch.Tensor) -> int:
    device = t.get_device()
    if device != _current_device():
        # the library works on the current device
        raise ValueError(f"tensor on {t.device}, current device is cuda:{_current_device()}")
    return _raw_stream(device)


def _check(status: int, what: str) -> None:
    if status != _lib.RDFFT_OK:
        raise RdfftError(status, what)


def rdfft_forward(buf: torch.Tensor) -> torch.Tensor:
    """In place: each row (last dim n) becomes its packed spectrum.  Returns ``buf``."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    _check(_lib.load().rdfft_forward(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf)), "rdfft_forward")
    return buf


def rdfft_inverse(buf: torch.Tensor) -> torch.Tensor:
    """In place: each packed spectrum row becomes its real signal.  Returns ``buf``."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    _check(_lib.load().rdfft_inverse(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf)), "rdfft_inverse")
    return buf


def rdfft_forward_halfcomplex(buf: torch.Tensor) -> torch.Tensor:
    """In place: each row becomes its packed spectrum in the halfcomplex layout.  Returns ``buf``."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    st = _lib.load().rdfft_forward_halfcomplex(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf))
    _check(st, "rdfft_forward_halfcomplex")
    return buf


def rdfft_inverse_halfcomplex(buf: torch.Tensor) -> torch.Tensor:
    """In place: each halfcomplex-layout spectrum row becomes its real signal.  Returns ``buf``."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    st = _lib.load().rdfft_inverse_halfcomplex(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf))
    _check(st, "rdfft_inverse_halfcomplex")
    return buf


def rdfft_pairs_to_halfcomplex(buf: torch.Tensor) -> torch.Tensor:
    """In place: each packed spectrum row moves from the pairs to the halfcomplex layout."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    st = _lib.load().rdfft_pairs_to_halfcomplex(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf))
    _check(st, "rdfft_pairs_to_halfcomplex")
    return buf


def rdfft_halfcomplex_to_pairs(buf: torch.Tensor) -> torch.Tensor:
    """In place: each packed spectrum row moves from the halfcomplex to the pairs layout."""
    n = buf.shape[-1]
    rows = buf.numel() // n if n else 0
    st = _lib.load().rdfft_halfcomplex_to_pairs(_dev(buf, "buf"), rows, n, _code(buf), _stream(buf))
    _check(st, "rdfft_halfcomplex_to_pairs")
    return buf


def _layer_shapes(x: torch.Tensor, c_spectra: torch.Tensor, out: torch.Tensor, out_name: str):
    """(q, kb, p, tokens) after checking that the tensors agree with each other.

    The library sees only pointers and sizes, so a tensor of the wrong shape, storage type
    or device would make it read or write outside that tensor; those are refused here.
    """
    if c_spectra.dim() != 3:
        raise ValueError(f"c_spectra must have shape (q, kb, p), got {tuple(c_spectra.shape)}")
    q, kb, p = c_spectra.shape
    xs = x.shape
    if len(xs) != 2 or xs[1] != kb * p:
        raise ValueError(f"x must have shape (tokens, {kb * p}), got {tuple(xs)}")
    tokens = xs[0]
    if out.shape != (tokens, q * p):
        raise ValueError(f"{out_name} must have shape ({tokens}, {q * p}), got {tuple(out.shape)}")
    dtype, device = x.dtype, x.get_device()
    if c_spectra.dtype != dtype or out.dtype != dtype or c_spectra.get_device() != device or out.get_device() != device:
        for name, t in (("c_spectra", c_spectra), (out_name, out)):
            if t.dtype != dtype:
                raise TypeError(f"{name} is {t.dtype}, x is {dtype}")
            if t.device != x.device:
                raise ValueError(f"{name} is on {t.device}, x on {x.device}")
    return q, kb, p, tokens


def _grad_shapes(x: torch.Tensor, dx: torch.Tensor, dc: torch.Tensor, cshape) -> None:
    """Refuses a dx unlike x, and a dc that is not float32 of the spectra's shape on x's device."""
    if dx.shape != x.shape or dx.dtype != x.dtype or dx.get_device() != x.get_device():
        raise ValueError(f"dx must match x: {tuple(x.shape)} {x.dtype} on {x.device}")
    if dc.shape != cshape or dc.get_device() != x.get_device():
        raise ValueError(f"dc must have shape {tuple(cshape)} on {x.device}, got {tuple(dc.shape)}")


def bca_forward(x: torch.Tensor, c_spectra: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
    """y[t] = W x[t] for the block-circulant W whose packed block spectra are ``c_spectra`` (q, kb, p)."""
    q, kb, p, tokens = _layer_shapes(x, c_spectra, y, "y")
    st = _lib.load().bca_forward(
        _dev(x, "x"), _dev(c_spectra, "c_spectra"), _dev(y, "y"), None,
        kb * p, q * p, p, tokens, _code(x), _stream(x),
    )
    _check(st, "bca_forward")
    return y


def bca_backward(x: torch.Tensor, c_spectra: torch.Tensor, gy: torch.Tensor, dx: torch.Tensor, dc: torch.Tensor):
    """Writes dL/dx into ``dx`` and dL/dc (float32, time domain, shape (q, kb, p)) into ``dc``.

    ``gy`` is left unspecified; ``dx`` may be ``gy`` itself when d_in == d_out (for blocks
    beyond 8192, with at most 8 blocks per row).
    """
    return _backward("bca_backward", x, c_spectra, gy, dx, dc)


def bca_backward_keep(x: torch.Tensor, c_spectra: torch.Tensor, gy: torch.Tensor, dx: torch.Tensor, dc: torch.Tensor):
    """``bca_backward`` that leaves ``gy`` as it was: ``dx`` apart from it, blocks of at most 8192."""
    return _backward("bca_backward_keep", x, c_spectra, gy, dx, dc)


def _backward(name, x, c_spectra, gy, dx, dc):
    q, kb, p, tokens = _layer_shapes(x, c_spectra, gy, "gy")
    _grad_shapes(x, dx, dc, (q, kb, p))
    if dc.dtype != torch.float32:
        raise TypeError("dc is float32")
    grads = _lib.BcaGrads(_dev(dx, "dx"), _dev(dc, "dc"))
    st = getattr(_lib.load(), name)(
        _dev(x, "x"), _dev(c_spectra, "c_spectra"), _dev(gy, "gy"), ctypes.byref(grads),
        kb * p, q * p, p, tokens, _code(x), _stream(x),
    )
    _check(st, name)
    return dx, dc


def _pointer_array(ts, name):
    if not all([t.is_cuda and t.is_contiguous() for t in ts]):
        for i, t in enumerate(ts):
            _dev(t, f"{name}[{i}]")  # raises for the first that is not
    return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])


def _batch_shapes(xs, cs, outs, out_name):
    if not (len(xs) == len(cs) == len(outs)):
        raise ValueError("one x, c_spectra and output per layer")
    first = _layer_shapes(xs[0], cs[0], outs[0], out_name)
    dtype, device = xs[0].dtype, xs[0].get_device()
    xshape, cshape, oshape = xs[0].shape, cs[0].shape, outs[0].shape
    for x, c, o in zip(xs, cs, outs):
        if (x.shape != xshape or c.shape != cshape or o.shape != oshape or x.dtype != dtype or c.dtype != dtype
                or o.dtype != dtype or x.get_device() != device or c.get_device() != device or o.get_device() != device):
            _layer_shapes(x, c, o, out_name)  # a layer that does not agree with itself has its own message
            raise ValueError("the layers of a batch share one shape, storage type and device")
    return first


def bca_forward_batched(xs, c_spectras, ys):
    """``bca_forward`` for several independent layers of one shape (lists of tensors), in one call."""
    if len(xs) == 0:
        return ys
    q, kb, p, tokens = _batch_shapes(xs, c_spectras, ys, "y")
    st = _lib.load().bca_forward_batched(
        len(xs), _pointer_array(xs, "x"), _pointer_array(c_spectras, "c_spectra"), _pointer_array(ys, "y"),
        kb * p, q * p, p, tokens, _code(xs[0]), _stream(xs[0]),
    )
    _check(st, "bca_forward_batched")
    return ys


def bca_backward_batched(xs, c_spectras, gys, dxs, dcs):
    """``bca_backward`` for several independent layers of one shape (lists of tensors), in one call."""
    if len(xs) == 0:
        return dxs, dcs
    q, kb, p, tokens = _batch_shapes(xs, c_spectras, gys, "gy")
    if not (len(dxs) == len(dcs) == len(xs)):
        raise ValueError("one dx and dc per layer")
    x0 = xs[0]
    shape, dtype, device, cshape = x0.shape, x0.dtype, x0.get_device(), c_spectras[0].shape
    for x, dx, dc in zip(xs, dxs, dcs):
        if dx.shape != shape or dx.dtype != dtype or dx.get_device() != device:
            raise ValueError(f"dx must match x: {tuple(x.shape)} {x.dtype} on {x.device}")
        if dc.shape != cshape or dc.get_device() != device or dc.dtype != torch.float32:
            raise ValueError(f"dc must be float32 of shape ({q}, {kb}, {p}) on {x.device}")
    grads = (_lib.BcaGrads * len(xs))(*zip(_pointer_array(dxs, "dx"), _pointer_array(dcs, "dc")))
    st = _lib.load().bca_backward_batched(
        len(xs), _pointer_array(xs, "x"), _pointer_array(c_spectras, "c_spectra"), _pointer_array(gys, "gy"), grads,
        kb * p, q * p, p, tokens, _code(xs[0]), _stream(xs[0]),
    )
    _check(st, "bca_backward_batched")
    return dxs, dcs


# -------------------------------------------------------------------------------------------------
# The operators around the adapter.  Tensors of the storage type are two-dimensional with
# consecutive elements in a row; a row stride of their own (a slice of wider rows) is fine.  A checkpoint is the
# pair (codes, scales): int8 (rows, n) and uint8 (rows, ceil(n / 32)).
#
# Each call goes through the native module, which takes the tensors as they are (a call's checks take 0.1 to 0.3 us
# there and 2 to 5 here); where that finds a tensor that is not what the call needs, what follows says so.

CHECKPOINT_BLOCK = 32
ACTIVATIONS = {"none": _lib.RDFFT_ACT_NONE, "relu": _lib.RDFFT_ACT_RELU, "gelu": _lib.RDFFT_ACT_GELU,
               "silu": _lib.RDFFT_ACT_SILU}


def _rows(t: torch.Tensor, name: str, dtype: torch.dtype, device: int, shape) -> tuple[int, int]:
    """(pointer, row stride) of a (rows, n) tensor of that type and device."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr(), shape[1]
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, is on {t.device}")
    rows, n = shape
    s0, s1 = t.stride()
    if (s1 != 1 and n > 1) or (s0 < n and rows > 1):
        raise ValueError(f"{name} must have consecutive elements in a row, and rows apart, got strides {t.stride()}")
    return t.data_ptr(), max(s0, n)


def _vector(t: torch.Tensor, name: str, dtype: torch.dtype, device: int, n: int) -> int:
    if t.dtype is dtype and t.shape == (n,) and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    if t.shape != (n,):
        raise ValueError(f"{name} must have shape ({n},), got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, is on {t.device}")
    raise ValueError(f"{name} must be contiguous")


def _first(t: torch.Tensor, name: str):
    """Pointer, row stride, (rows, n), storage type, its code, device and stream of a call's first tensor."""
    shape, dtype, device = t.shape, t.dtype, t.get_device()
    code = _CODES.get(dtype)
    if len(shape) != 2 or code is None or device < 0 or device != _current_device():
        if len(shape) != 2:
            raise ValueError(f"{name} must be two-dimensional, got shape {tuple(shape)}")
        if device < 0:
            raise ValueError(f"{name} must be a device tensor")
        _code(t), _stream(t)  # (one of them raises)
    if t.is_contiguous():
        return t.data_ptr(), shape[1], shape, dtype, code, device, _raw_stream(device)
    return (*_rows(t, name, dtype, device, shape), shape, dtype, code, device, _raw_stream(device))


def _held(checkpoint, device: int, rows: int, n: int) -> tuple[int, int]:
    """Pointers of a (codes, scales) pair for (rows, n) values."""
    codes, scales = checkpoint
    if codes is None or scales is None:
        raise ValueError("a checkpoint is the pair (codes, scales), and one of them is None")
    blocks = -(-n // CHECKPOINT_BLOCK)
    if (codes.dtype is torch.int8 and scales.dtype is torch.uint8 and codes.shape == (rows, n)
            and scales.shape == (rows, blocks) and codes.get_device() == device and scales.get_device() == device
            and codes.is_contiguous() and scales.is_contiguous()):
        return codes.data_ptr(), scales.data_ptr()
    # which of these it is
    for name, t, dtype, shape in (("codes", codes, torch.int8, (rows, n)), ("scales", scales, torch.uint8, (rows, blocks))):
        if t.dtype is not dtype:
            raise TypeError(f"a checkpoint's {name} are {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
        if t.get_device() != device:
            raise ValueError(f"{name} must be on cuda:{device}, is on {t.device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _scratch(need: int, given, device: int, what: str):
    """(tensor to keep alive, pointer, bytes) of a workspace; one is allocated if none is given."""
    if need == 0:
        return None, 0, 0
    if given is None:
        given = torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", device))
    elif given.get_device() != device or not given.is_contiguous():
        raise ValueError(f"the workspace must be a contiguous tensor on cuda:{device}")
    size = given.numel() * given.element_size()
    if size < need:
        raise ValueError(f"the workspace has {size} bytes, {what} needs {need}")
    return given, given.data_ptr(), size


# (the sizes of workspaces follow from their arguments alone)
@functools.lru_cache(maxsize=4096)
def _need(name: str, *args: int) -> int:
    need = int(getattr(_lib.load(), name)(*args))
    if need < 0:
        _check(need, name)
    return need


def checkpoint_like(x: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """An empty 8-bit checkpoint (codes, scales) for the values of a (rows, n) tensor."""
    rows, n = x.shape
    return (torch.empty((rows, n), dtype=torch.int8, device=x.device),
            torch.empty((rows, -(-n // CHECKPOINT_BLOCK)), dtype=torch.uint8, device=x.device))


def act8_quantize(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor):
    """The 8-bit checkpoint of x (rows, n): int8 codes, and one scale byte for 32 values of a row."""
    status = None
    if x.is_cuda:
        device = _current_device()
        status = _lib.binding().act8_quantize(x, codes, scales, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(x, "x")
        rows, n = shape
        held = _lib.pack["act8"](*_held((codes, scales), device, rows, n))
        status = _lib.load().act8_quantize(p, ld, held, rows, n, code, stream)
    if status:
        _check(status, "act8_quantize")
    return codes, scales


def act8_dequantize(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """What a checkpoint stands for, in ``out``'s type (exact in float32 and bfloat16)."""
    status = None
    if out.is_cuda:
        device = _current_device()
        status = _lib.binding().act8_dequantize(codes, scales, out, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(out, "out")
        rows, n = shape
        held = _lib.pack["act8"](*_held((codes, scales), device, rows, n))
        status = _lib.load().act8_dequantize(held, p, ld, rows, n, code, stream)
    if status:
        _check(status, "act8_dequantize")
    return out


_F32 = torch.float32
_NONE = (None, None)


def layer_norm_forward(x, weight, bias, y, *, residual=None, mean=None, rstd=None, checkpoint=None, eps=1e-5):
    """y = norm(x (+ residual)) * weight (+ bias) per row; weight, bias, mean and rstd are float32.

    ``mean`` and ``rstd`` (rows,) and ``checkpoint``, of the norm's input, are written if given.
    ``y`` may be ``x`` or ``residual``.
    """
    status = None
    if x.is_cuda:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        status = _lib.binding().layer_norm_forward(x, residual, weight, bias, y, mean, rstd, codes, scales, eps, device,
                                                   _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(x, "x")
        rows, n = shape
        a = _lib.pack["layer_norm_forward"](
            p, ld,
            *((0, 0) if residual is None else _rows(residual, "residual", dtype, device, shape)),
            _vector(weight, "weight", _F32, device, n),
            0 if bias is None else _vector(bias, "bias", _F32, device, n),
            *_rows(y, "y", dtype, device, shape),
            0 if mean is None else _vector(mean, "mean", _F32, device, rows),
            0 if rstd is None else _vector(rstd, "rstd", _F32, device, rows),
            *((0, 0) if checkpoint is None else _held(checkpoint, device, rows, n)))
        status = _lib.load().layer_norm_forward(a, rows, n, eps, code, stream)
    if status:
        _check(status, "layer_norm_forward")
    return y


def layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, *, residual=None, workspace=None):
    """Writes the norm's gradients: dx (of x and of the residual alike), and float32 dweight and dbias.

    ``x`` is the forward's x, or the checkpoint (codes, scales) of the norm's input; ``dx`` may be ``dy``.
    ``workspace``: ``layer_norm_backward_workspace(rows, n)`` bytes, allocated if not given.
    """
    status = None
    values = isinstance(x, torch.Tensor)
    if not values and residual is not None:
        raise ValueError("a checkpoint is of the norm's input, residual included")
    if dy.is_cuda:
        device = _current_device()
        codes, scales = _NONE if values else x
        status = _lib.binding().layer_norm_backward(dy, x if values else None, residual, codes, scales, weight, mean, rstd,
                                                    dx, dweight, dbias, workspace, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(dy, "dy")
        rows, n = shape
        if values:
            inputs = (*_rows(x, "x", dtype, device, shape),
                      *((0, 0) if residual is None else _rows(residual, "residual", dtype, device, shape)), 0, 0)
        else:
            inputs = (0, 0, 0, 0, *_held(x, device, rows, n))
        keep, scratch, size = _scratch(_need("layer_norm_backward_workspace", rows, n), workspace, device,
                                       "layer_norm_backward")
        a = _lib.pack["layer_norm_backward"](
            p, ld, *inputs, _vector(weight, "weight", _F32, device, n), _vector(mean, "mean", _F32, device, rows),
            _vector(rstd, "rstd", _F32, device, rows), *_rows(dx, "dx", dtype, device, shape),
            _vector(dweight, "dweight", _F32, device, n), _vector(dbias, "dbias", _F32, device, n), scratch, size)
        status = _lib.load().layer_norm_backward(a, rows, n, code, stream)
    if status:
        _check(status, "layer_norm_backward")
    return dx, dweight, dbias


def layer_norm_backward_workspace(rows: int, n: int) -> int:
    """Bytes of workspace that ``layer_norm_backward`` needs."""
    return _need("layer_norm_backward_workspace", rows, n)


def _activation(name: str) -> int:
    act = ACTIVATIONS.get(name)
    if act is None:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, got {name!r}")
    return act


def linear_forward(x, w, y, *, bias=None, activation="none", residual=None, checkpoint=None, workspace=None):
    """y = act(x w^T + bias) + residual, with x (tokens, d_in), w (d_out, d_in) and the rest of one storage type.

    ``checkpoint``, of the pre-activation, is written if given.  ``y`` may be ``residual``.
    ``workspace``: ``linear_forward_workspace(...)`` bytes, allocated if not given.
    """
    status = None
    act = ACTIVATIONS.get(activation)
    if x.is_cuda and act is not None:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        status = _lib.binding().linear_forward(x, w, bias, residual, y, codes, scales, act, workspace, device,
                                               _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(x, "x")
        tokens, d_in = shape
        d_out = w.shape[0]
        act = _activation(activation)
        out = (tokens, d_out)
        keep, scratch, size = _scratch(_need("linear_forward_workspace", d_in, d_out, tokens, code), workspace, device,
                                       "linear_forward")
        a = _lib.pack["linear_forward"](
            p, ld, *_rows(w, "w", dtype, device, (d_out, d_in)),
            0 if bias is None else _vector(bias, "bias", dtype, device, d_out),
            *((0, 0) if residual is None else _rows(residual, "residual", dtype, device, out)),
            *_rows(y, "y", dtype, device, out),
            *((0, 0) if checkpoint is None else _held(checkpoint, device, tokens, d_out)), scratch, size)
        status = _lib.load().linear_forward(a, d_in, d_out, tokens, act, code, stream)
    if status:
        _check(status, "linear_forward")
    return y


def linear_forward_workspace(d_in: int, d_out: int, tokens: int, dtype: torch.dtype) -> int:
    """Bytes of workspace that ``linear_forward`` needs (0: none)."""
    return _need("linear_forward_workspace", d_in, d_out, tokens, _CODES[dtype])


def linear_backward(dy, x, w, *, dx=None, dw=None, db=None, activation="none", checkpoint=None, add=None,
                    workspace=None):
    """Writes those of dx = dz w (+ add), dw = dz^T x and db = sum of dz that are given, dz = dy act'(z).

    z is what ``checkpoint`` stands for (not needed without an activation).  relu's slope at a positive value that its block
    holds as zero is 0: for normal z that puts dz 0.11 of its norm off the gradient at z itself (gelu and silu less
    than 0.01).  ``x`` may be None without dw, ``w`` without dx; ``dx`` may be ``add``.  ``workspace``: ``linear_backward_workspace(...)`` bytes, allocated if not given.
    """
    status = None
    act = ACTIVATIONS.get(activation)
    if dy.is_cuda and act is not None:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        status = _lib.binding().linear_backward(dy, x, w, dx, dw, db, add, codes, scales, act, workspace, device,
                                                _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(dy, "dy")
        tokens, d_out = shape
        act = _activation(activation)
        d_in = 1  # (db alone)
        if dx is not None:
            if w is None:
                raise ValueError("dx needs w")
            d_in = dx.shape[-1]
        if dw is not None:
            if x is None:
                raise ValueError("dw needs x")
            if dx is not None and dw.shape[-1] != d_in:
                raise ValueError(f"dx and dw have {d_in} and {dw.shape[-1]} columns")
            d_in = dw.shape[-1]
        held = (0, 0)
        if act != _lib.RDFFT_ACT_NONE:
            if checkpoint is None:
                raise ValueError(f"the gradient through {activation} needs the checkpoint of the pre-activation")
            held = _held(checkpoint, device, tokens, d_out)
        none = (0, 0)
        keep, scratch, size = _scratch(
            _need("linear_backward_workspace", d_in, d_out, tokens, dx is not None, dw is not None, db is not None, act, code),
            workspace, device, "linear_backward")
        a = _lib.pack["linear_backward"](
            p, ld, *held,
            *(none if dw is None else _rows(x, "x", dtype, device, (tokens, d_in))),
            *(none if dx is None else _rows(w, "w", dtype, device, (d_out, d_in))),
            *(none if dx is None or add is None else _rows(add, "add", dtype, device, (tokens, d_in))),
            *(none if dx is None else _rows(dx, "dx", dtype, device, (tokens, d_in))),
            *(none if dw is None else _rows(dw, "dw", dtype, device, (d_out, d_in))),
            0 if db is None else _vector(db, "db", dtype, device, d_out), scratch, size)
        status = _lib.load().linear_backward(a, d_in, d_out, tokens, act, code, stream)
    if status:
        _check(status, "linear_backward")
    return dx, dw, db


def linear_backward_workspace(d_in: int, d_out: int, tokens: int, dtype: torch.dtype, activation: str = "none", *,
                              dx: bool = True, dw: bool = True, db: bool = True) -> int:
    """Bytes of workspace that ``linear_backward`` needs for the gradients that are wanted."""
    return _need("linear_backward_workspace", d_in, d_out, tokens, dx, dw, db, _activation(activation), _CODES[dtype])


FP8_BLOCK = 128
_FP8 = torch.float8_e4m3fn


def _held8(held, device: int, rows: int, n: int, what: str) -> tuple[int, int, int, int, int]:
    """Pointers and row strides of a (codes, scales) pair in 8-bit floating point for (rows, n) values, and its block_rows."""
    codes, scales = held
    if codes is None or scales is None:
        raise ValueError(f"{what} is the pair (codes, scales), and one of them is None")
    blocks, bands = -(-n // FP8_BLOCK), -(-rows // FP8_BLOCK)
    if scales.dim() != 2 or scales.shape[1] != blocks or scales.shape[0] not in (rows, bands):
        raise ValueError(f"the scales of {what} must have shape {(rows, blocks)}, or {(bands, blocks)} in tiles, "
                         f"got {tuple(scales.shape)}")
    return (*_rows(codes, f"codes of {what}", _FP8, device, (rows, n)),
            *_rows(scales, f"scales of {what}", torch.uint8, device, tuple(scales.shape)),
            1 if scales.shape[0] == rows else FP8_BLOCK)


def fp8_like(x: torch.Tensor, *, columns: bool = False, tiles: bool = False) -> tuple[torch.Tensor, torch.Tensor]:
    """Empty (codes, scales) in 8-bit floating point for a (rows, n) tensor, or for its ``columns`` (its transpose).

    A scale is for 128 consecutive values of a row or, with ``tiles``, for 128 x 128.
    """
    rows, n = reversed(x.shape) if columns else x.shape
    blocks, bands = -(-n // FP8_BLOCK), -(-rows // FP8_BLOCK) if tiles else rows
    codes = torch.empty((rows, -(-n // 16) * 16), dtype=_FP8, device=x.device)
    scales = torch.empty((bands, -(-blocks // 4) * 4), dtype=torch.uint8, device=x.device)
    return codes[:, :n], scales[:, :blocks]


def fp8_quantize(x: torch.Tensor, held=None, *, columns=None):
    """Writes x (rows, n) in 8-bit floating point into ``held`` (codes, scales), and its transpose into ``columns``.

    The shape of the scales says whether a scale is for 128 values of a row or for a tile of 128 x 128.
    """
    if held is None and columns is None:
        raise ValueError("fp8_quantize needs held or columns to write to")
    status = None
    if x.is_cuda:
        device = _current_device()
        status = _lib.binding().fp8_quantize(x, *(held or _NONE), *(columns or _NONE), device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(x, "x")
        rows, n = shape
        to = None if held is None else _lib.pack["fp8"](*_held8(held, device, rows, n, "held"))
        across = None if columns is None else _lib.pack["fp8"](*_held8(columns, device, n, rows, "columns"))
        status = _lib.load().fp8_quantize(p, ld, to, across, rows, n, code, stream)
    if status:
        _check(status, "fp8_quantize")
    return held, columns


def fp8_dequantize(held, out: torch.Tensor) -> torch.Tensor:
    """What (codes, scales) in 8-bit floating point stand for, in ``out``'s type: exact in float32, and in bfloat16 but for the
    smallest codes of the smallest scales, which need bits below its 2^-133."""
    status = None
    if out.is_cuda:
        device = _current_device()
        status = _lib.binding().fp8_dequantize(*held, out, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(out, "out")
        rows, n = shape
        status = _lib.load().fp8_dequantize(_lib.pack["fp8"](*_held8(held, device, rows, n, "held")), p, ld, rows, n, code,
                                            stream)
    if status:
        _check(status, "fp8_dequantize")
    return out


def rms_norm_forward(x, weight, y=None, *, residual=None, summed=None, rstd=None, checkpoint=None, y8=None, eps=1e-6):
    """y = u / sqrt(mean(u^2) + eps) * weight per row, u = x (+ residual) rounded to x's type; weight and rstd are float32.

    Written if given: ``y``, ``y8`` (codes, scales), which is y in 8-bit floating point, ``summed``, which is u, ``rstd``
    (rows,), and ``checkpoint``, of u.  ``y`` and ``summed`` may be ``x`` or ``residual``.
    """
    status = None
    if x.is_cuda:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        codes8, scales8 = _NONE if y8 is None else y8
        status = _lib.binding().rms_norm_forward(x, residual, weight, y, summed, rstd, codes, scales, codes8, scales8, eps,
                                                 device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(x, "x")
        rows, n = shape
        none = (0, 0)
        a = _lib.pack["rms_norm_forward"](
            p, ld,
            *(none if residual is None else _rows(residual, "residual", dtype, device, shape)),
            _vector(weight, "weight", _F32, device, n),
            *(none if y is None else _rows(y, "y", dtype, device, shape)),
            *(none if summed is None else _rows(summed, "summed", dtype, device, shape)),
            0 if rstd is None else _vector(rstd, "rstd", _F32, device, rows),
            *(none if checkpoint is None else _held(checkpoint, device, rows, n)),
            *((0, 0, 0, 0, 0) if y8 is None else _held8(y8, device, rows, n, "y8")))
        status = _lib.load().rms_norm_forward(a, rows, n, eps, code, stream)
    if status:
        _check(status, "rms_norm_forward")
    return y


def rms_norm_backward(dy, u, weight, rstd, dx, dweight=None, *, add=None, workspace=None):
    """Writes the norm's gradients: dx (+ ``add``), of x and of the residual alike, and float32 dweight if given.

    ``u`` is what the forward left in ``summed`` (x itself without a residual), or its checkpoint (codes, scales); ``add`` a
    gradient that reaches the sum another way.  ``dx`` may be ``dy`` or ``add``.
    ``workspace``: ``rms_norm_backward_workspace(rows, n)`` bytes, allocated if not given (none without dweight).
    """
    status = None
    values = isinstance(u, torch.Tensor)
    if dy.is_cuda:
        device = _current_device()
        codes, scales = _NONE if values else u
        status = _lib.binding().rms_norm_backward(dy, u if values else None, codes, scales, weight, rstd, add, dx, dweight,
                                                  workspace, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(dy, "dy")
        rows, n = shape
        inputs = (*_rows(u, "u", dtype, device, shape), 0, 0) if values else (0, 0, *_held(u, device, rows, n))
        keep, scratch, size = None, 0, 0
        if dweight is not None:
            keep, scratch, size = _scratch(_need("rms_norm_backward_workspace", rows, n), workspace, device,
                                           "rms_norm_backward")
        a = _lib.pack["rms_norm_backward"](
            p, ld, *inputs, _vector(weight, "weight", _F32, device, n), _vector(rstd, "rstd", _F32, device, rows),
            *((0, 0) if add is None else _rows(add, "add", dtype, device, shape)), *_rows(dx, "dx", dtype, device, shape),
            0 if dweight is None else _vector(dweight, "dweight", _F32, device, n), scratch, size)
        status = _lib.load().rms_norm_backward(a, rows, n, code, stream)
    if status:
        _check(status, "rms_norm_backward")
    return dx, dweight


def rms_norm_backward_workspace(rows: int, n: int) -> int:
    """Bytes of workspace that ``rms_norm_backward`` needs for dweight."""
    return _need("rms_norm_backward_workspace", rows, n)


def linear_fp8_forward(x, w, y, *, bias=None, activation="none", residual=None, checkpoint=None, workspace=None):
    """y = act(x w^T + bias) + residual, with x (tokens, d_in) and w (d_out, d_in) as (codes, scales) in 8-bit floating point.

    bias, residual and y are of one storage type.  ``checkpoint``, of the pre-activation, is written if given.  ``y`` may be
    ``residual``.  ``workspace``: ``linear_fp8_forward_workspace(...)`` bytes, allocated if not given.
    """
    status = None
    act = ACTIVATIONS.get(activation)
    if y.is_cuda and act is not None:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        status = _lib.binding().linear_fp8_forward(*x, *w, bias, residual, y, codes, scales, act, workspace, device,
                                                   _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(y, "y")
        tokens, d_out = shape
        d_in = w[0].shape[-1]
        act = _activation(activation)
        keep, scratch, size = _scratch(_need("linear_fp8_forward_workspace", d_in, d_out, tokens, code), workspace, device,
                                       "linear_fp8_forward")
        a = _lib.pack["linear_fp8_forward"](
            *_held8(x, device, tokens, d_in, "x"), *_held8(w, device, d_out, d_in, "w"),
            0 if bias is None else _vector(bias, "bias", dtype, device, d_out),
            *((0, 0) if residual is None else _rows(residual, "residual", dtype, device, shape)), p, ld,
            *((0, 0) if checkpoint is None else _held(checkpoint, device, tokens, d_out)), scratch, size)
        status = _lib.load().linear_fp8_forward(a, d_in, d_out, tokens, act, code, stream)
    if status:
        _check(status, "linear_fp8_forward")
    return y


def linear_fp8_forward_workspace(d_in: int, d_out: int, tokens: int, dtype: torch.dtype) -> int:
    """Bytes of workspace that ``linear_fp8_forward`` needs (0: none)."""
    return _need("linear_fp8_forward_workspace", d_in, d_out, tokens, _CODES[dtype])


def linear_fp8_backward(dy, x, w, *, dx=None, dw=None, db=None, activation="none", checkpoint=None, add=None,
                        workspace=None):
    """Writes those of dx = dz w (+ add), dw = dz^T x and db = sum of dz that are given, dz = dy act'(z) in 8 bits.

    ``x`` (d_in, tokens) and ``w`` (d_in, d_out) are what ``fp8_quantize`` leaves in ``columns`` of x and W; ``x`` may be None
    without dw, ``w`` without dx.  z is what ``checkpoint`` stands for (not needed without an activation; relu's slope at a
    positive value that its block holds as zero is 0, as in ``linear_backward``).  ``dx`` may be ``add``.
    ``workspace``: ``linear_fp8_backward_workspace(...)`` bytes, allocated if not given.
    """
    status = None
    act = ACTIVATIONS.get(activation)
    if dy.is_cuda and act is not None:
        device = _current_device()
        codes, scales = _NONE if checkpoint is None else checkpoint
        status = _lib.binding().linear_fp8_backward(dy, *(_NONE if x is None else x), *(_NONE if w is None else w), dx, dw, db,
                                                    add, codes, scales, act, workspace, device, _raw_stream(device))
    if status is None:
        p, ld, shape, dtype, code, device, stream = _first(dy, "dy")
        tokens, d_out = shape
        act = _activation(activation)
        d_in = 1  # (db alone)
        if dx is not None:
            if w is None:
                raise ValueError("dx needs w")
            d_in = dx.shape[-1]
        if dw is not None:
            if x is None:
                raise ValueError("dw needs x")
            if dx is not None and dw.shape[-1] != d_in:
                raise ValueError(f"dx and dw have {d_in} and {dw.shape[-1]} columns")
            d_in = dw.shape[-1]
        held = (0, 0)
        if act != _lib.RDFFT_ACT_NONE:
            if checkpoint is None:
                raise ValueError(f"the gradient through {activation} needs the checkpoint of the pre-activation")
            held = _held(checkpoint, device, tokens, d_out)
        none, none8 = (0, 0), (0, 0, 0, 0, 0)
        keep, scratch, size = _scratch(
            _need("linear_fp8_backward_workspace", d_in, d_out, tokens, dx is not None, dw is not None, db is not None, code),
            workspace, device, "linear_fp8_backward")
        a = _lib.pack["linear_fp8_backward"](
            p, ld, *held,
            *(none8 if dw is None else _held8(x, device, d_in, tokens, "x")),
            *(none8 if dx is None else _held8(w, device, d_in, d_out, "w")),
            *(none if dx is None or add is None else _rows(add, "add", dtype, device, (tokens, d_in))),
            *(none if dx is None else _rows(dx, "dx", dtype, device, (tokens, d_in))),
            *(none if dw is None else _rows(dw, "dw", dtype, device, (d_out, d_in))),
            0 if db is None else _vector(db, "db", dtype, device, d_out), scratch, size)
        status = _lib.load().linear_fp8_backward(a, d_in, d_out, tokens, act, code, stream)
    if status:
        _check(status, "linear_fp8_backward")
    return dx, dw, db


def linear_fp8_backward_workspace(d_in: int, d_out: int, tokens: int, dtype: torch.dtype, *, dx: bool = True, dw: bool = True,
                                  db: bool = True) -> int:
    """Bytes of workspace that ``linear_fp8_backward`` needs for the gradients that are wanted."""
    return _need("linear_fp8_backward_workspace", d_in, d_out, tokens, dx, dw, db, _CODES[dtype])


def rdfft_init() -> None:
    _check(_lib.load().rdfft_init(), "rdfft_init")


def rdfft_table_bytes() -> int:
    return int(_lib.load().rdfft_table_bytes())
