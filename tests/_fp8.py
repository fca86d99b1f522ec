"""The 8-bit floating point format and the products of its operands in 64 bits, on the CPU, for the tests.

A value is held as the e4m3 number nearest to x / 2^e (ties to the even code), 2^e the least power of two with
max|x| <= 448 * 2^e over its block: 128 values of a row, or a tile of 128 x 128.
"""

from __future__ import annotations

import numpy as np
import torch

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _table():
    """The 127 numbers >= 0 of e4m3, by code."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m / 8.0 * 2.0**-6, (1 + m / 8.0) * 2.0 ** (e - 7.0))


TABLE = _table()


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """Codes (uint8) of float64 values of at most 448 in size."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(TABLE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = TABLE[hi] - a, a - TABLE[lo]
    take_lo = (down < up) | ((down == up) & (lo % 2 == 0))
    return (np.where(take_lo, lo, hi) | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def encode(x: np.ndarray, tiles: bool = False):
    """(codes, scale bytes) of float64 rows."""
    rows, n = x.shape
    high = BLOCK if tiles else 1
    blocks, bands = -(-n // BLOCK), -(-rows // high)
    v = np.zeros((bands * high, blocks * BLOCK))
    v[:rows, :n] = x
    v = v.reshape(bands, high, blocks, BLOCK)
    top = np.abs(v).max(axis=(1, 3))  # (NaN if there is one)
    fine = np.isfinite(top)
    m, k = np.frexp(np.where(fine, top, 1.0))
    e = np.where(m <= 0.875, k - 9, k - 8)
    e = np.maximum(np.where(top == 0, -127, e), -127)
    with np.errstate(invalid="ignore"):
        codes = round_e4m3(np.where(fine[:, None, :, None], v, 0.0) * np.exp2(-e.astype(float))[:, None, :, None])
    codes = np.where(fine[:, None, :, None], codes, 0x7F).astype(np.uint8)
    return codes.reshape(bands * high, blocks * BLOCK)[:rows, :n], np.where(fine, e + 127, 255).astype(np.uint8)


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    rows, n = codes.shape
    size = np.append(TABLE, np.nan)[codes & 127]
    value = np.where(codes >= 128, -size, size)
    power = np.where(scales == 255, np.nan, np.exp2(scales.astype(float) - 127))
    power = power if scales.shape[0] == rows else np.repeat(power, BLOCK, axis=0)[:rows]
    return value * np.repeat(power, BLOCK, axis=1)[:, :n]


def host(held):
    """(codes, scales) on the host as uint8 arrays."""
    return held[0].view(torch.uint8).cpu().numpy(), held[1].cpu().numpy()


def value(held) -> np.ndarray:
    return decode(*host(held))


def f64(t) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def room(rows, n, tiles=False, pad=0, junk=True, device="cuda"):
    """(codes, scales) of wider rows, whose every byte is junk (NaN codes, NaN scales)."""
    blocks, bands = -(-n // BLOCK), -(-rows // BLOCK) if tiles else rows
    codes = torch.full((rows, -(-n // 16) * 16 + 16 * pad), 0x7F if junk else 0, dtype=torch.uint8, device=device)
    scales = torch.full((bands, -(-blocks // 4) * 4 + 4 * pad), 255 if junk else 0, dtype=torch.uint8, device=device)
    return codes.view(torch.float8_e4m3fn)[:, :n], scales[:, :blocks]


def random_operand(rows, n, seed, tiles=False, pad=0, spread=3):
    """An operand made on the host: normal values, blocks of different sizes."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, n)) * np.exp2(rng.integers(-spread, spread + 1, (rows, 1)))
    x *= np.exp2(rng.integers(-spread, spread + 1, -(-n // BLOCK)))[np.arange(n) // BLOCK]
    held = room(rows, n, tiles, pad)
    for to, a in zip(held, encode(x, tiles)):
        to.view(torch.uint8).copy_(torch.from_numpy(a))
    return held


# a rounding to the storage type: half a step of the largest value of a binade, and its root mean square at most
UNIT = {"f32": 2.0**-24, "bf16": 2.0**-8, "f16": 2.0**-11}


def matmul64(a: np.ndarray, b: np.ndarray) -> np.ndarray:
    """a b^T in float64."""
    if a.shape[0] * b.shape[0] * a.shape[1] < 1 << 24 or not torch.cuda.is_available():
        return a @ b.T
    return (torch.from_numpy(a).cuda() @ torch.from_numpy(np.ascontiguousarray(b.T)).cuda()).cpu().numpy()


def product_error(got: np.ndarray, a: np.ndarray, b: np.ndarray, dtype: str, more=0.0, slope=1.0, what=""):
    """Checks got against (a b^T, or `more`'s function of it), a (m, k) and b (n, k) being what the operands stand for.

    16-bit results: of the 64 products that an instruction adds, each is off by at most 2^-16 of the largest p, so their
    sum by 2^-10 |p|, and the sums of k / 64 instructions by 2^-10 sqrt(k / 64) times the 2-norm of an output's products;
    over all outputs these are of either sign and leave less than 1e-4 of the norm.  `slope` bounds how much of a
    difference a function of the product passes on.  float32 results: 2^-24 for every addition, in runs of k, taken as random:
    2^-22 sqrt(k) of the products' 2-norm at most.  A rounding to the type: UNIT of the value, 0.6 of that over all.
    """
    z = matmul64(a, b)
    want = more(z) if callable(more) else z + more
    k = a.shape[1]
    size = np.sqrt(matmul64(a * a, b * b))
    drop = 2.0**-22 * np.sqrt(max(k, 1)) if dtype == "f32" else 2.0**-10 * np.sqrt(-(-k // 64))
    tiny = 2.0**-25 if dtype == "f16" else 0.0  # (half a step of float16's smallest numbers)
    bound = UNIT[dtype] * np.abs(want) * 1.01 + slope * drop * size + 2.0**-22 * np.abs(want) + tiny
    if dtype == "f16":
        # what lies past 65504 by more than an output may be off is infinite there, up to it by less may be
        sure = np.abs(want) - bound >= 65520
        past = np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + bound >= 65520)
        assert past[sure].all(), what
        got, want = np.where(past, 0.0, got), np.where(past, 0.0, want)
    off = np.abs(got - want)
    assert np.isfinite(got).all(), what
    bad = off > bound
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size}, first {np.argwhere(bad)[0]}: {got[bad][0]!r} "
                           f"for {want[bad][0]!r}, bound {bound[bad][0]!r}")
    norm = np.linalg.norm(want)
    if norm > 0 and dtype != "f16" or norm > 1e-2:
        rel = np.linalg.norm(off) / norm
        assert rel <= 0.6 * UNIT[dtype] + (1e-6 if dtype == "f32" else 1e-4 * max(1.0, slope * np.linalg.norm(size) / norm)), (what, rel)
