"""Plain 64-bit definitions of the low-bit matrix operators, and their storage,
in numpy: what the tests compare with."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def ceil_div(a: int, b: int) -> int:
    return -(-a // b)


def sizes(fmt: str, rows: int, cols: int):
    b = ceil_div(cols, 32)
    if fmt == "e2m1":
        return 16 * b, rows * 16 * b, ceil_div(rows, 128) * ceil_div(b, 4) * 512
    return 32 * b, rows * 32 * b, rows * ceil_div(b, 8) * 8


def quantize(fmt: str, x: np.ndarray):
    """(codes, scale bytes) of x: codes (rows, 32 blocks) as 4-bit codes or
    signed integers, scale bytes (rows, blocks)."""
    rows, cols = x.shape
    nb = ceil_div(cols, 32)
    a = np.zeros((rows, nb * 32))
    a[:, :cols] = x
    a = a.reshape(rows, nb, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(a).max(-1)
    finite = np.isfinite(a).all(-1)
    _, e = np.frexp(np.where(finite, top, 1.0))
    E = np.where(top == 0, -127, e - 1 - (2 if fmt == "e2m1" else 0)).clip(-127, 127)
    s = np.where(finite, E + 127, 255).astype(np.uint8)
    v = np.where(finite[..., None], a, 0.0) * np.exp2(-E.astype(np.float64))[..., None]
    if fmt == "i8":
        return np.rint(v * 64).clip(-127, 127).astype(np.int8).reshape(rows, -1), s
    d = np.abs(np.abs(v)[..., None] - GRID)
    near = d == d.min(-1, keepdims=True)
    lo = near.argmax(-1)
    hi = 7 - near[..., ::-1].argmax(-1)
    code = np.where(lo % 2 == 0, lo, hi)  # of two equally near ones the even code
    # a value that rounds to zero keeps its sign, as a zero does
    return (code + 8 * np.signbit(v)).astype(np.uint8).reshape(rows, -1), s


def values(fmt: str, codes: np.ndarray, scales: np.ndarray, cols: int) -> np.ndarray:
    rows = codes.shape[0]
    if fmt == "i8":
        v = codes.astype(np.float64) / 64
    else:
        v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v.reshape(rows, -1, 32) * unit[..., None]).reshape(rows, -1)[:, :cols]


def rounded(fmt: str, x: np.ndarray) -> np.ndarray:
    return values(fmt, *quantize(fmt, x), x.shape[1])


def scale_index(fmt: str, rows: int, cols: int) -> np.ndarray:
    """Byte of the scale of block j of row i."""
    nb = ceil_div(cols, 32)
    i, j = np.arange(rows)[:, None], np.arange(nb)[None, :]
    if fmt == "i8":
        return i * (ceil_div(nb, 8) * 8) + j
    tile = (i // 128) * ceil_div(nb, 4) + j // 4
    return tile * 512 + i % 32 * 16 + i % 128 // 32 * 4 + j % 4


def pack(fmt: str, codes: np.ndarray, scales: np.ndarray, cols: int, ld: int | None = None, fill: int = 0):
    """(code bytes, scale bytes) in storage order; unused bytes hold `fill`,
    E2M1's scales past the last block 0."""
    rows = codes.shape[0]
    least, _, nscale = sizes(fmt, rows, cols)
    ld = least if ld is None else ld
    out = np.full((rows, ld), fill, np.uint8)
    if fmt == "i8":
        out[:, :least] = codes.view(np.uint8)
    else:
        out[:, :least] = codes[:, 0::2] | codes[:, 1::2] << 4
    sc = np.full(nscale, fill, np.uint8)
    if fmt == "e2m1":
        padded = ceil_div(ceil_div(cols, 32), 4) * 128
        sc[scale_index(fmt, rows, padded)] = 0
    sc[scale_index(fmt, rows, cols)] = scales
    return out, sc


_erf = np.vectorize(math.erf, otypes=[float])


def act(name: str, x: np.ndarray):
    """act(x) and act'(x)."""
    with np.errstate(over="ignore"):
        if name == "silu":
            s = 1 / (1 + np.exp(-x))
            return x * s, s * (1 + x * (1 - s))
        if name == "gelu":
            c = 0.5 * (1 + _erf(x / math.sqrt(2)))
            return x * c, c + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return np.where(x > 0, x, np.where(np.isnan(x), x, 0.0)), np.where(np.isnan(x), x, (x > 0) * 1.0)


def bf16(x: np.ndarray) -> np.ndarray:
    """x (float32) rounded to bf16 values."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().float().numpy()
