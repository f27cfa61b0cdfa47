"""Plain float64 forms of the microscaled operators, shared by their tests (not
a test module).  Written from the formats' definitions with numpy; nothing here
calls the library."""
from __future__ import annotations

import numpy as np

FP8, FP4 = 0, 1
BLOCK = 32
EMAX = {FP8: 8, FP4: 2}
TOP = {FP8: 448.0, FP4: 6.0}
F4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def _f8_table():
    t = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = np.nan if (c & 127) == 127 else np.ldexp(m / 8, -6) if e == 0 else np.ldexp(1 + m / 8, e - 7)
        t[c] = -v if c & 128 else v
    return t


F8 = _f8_table()


def quantize(x, fmt):
    """(codes one per value [..., K], scales [..., K / 32]) of float64 x."""
    x = np.asarray(x, np.float64)
    t = x.reshape(*x.shape[:-1], -1, BLOCK)
    finite = np.isfinite(t).all(-1)
    top = np.where(finite, np.abs(np.where(np.isfinite(t), t, 0)).max(-1), 0)
    e = np.frexp(top)[1].astype(np.int64) - 1 - EMAX[fmt]
    e = np.where(top == 0, -127, np.clip(e, -127, 127))
    z = np.where(finite[..., None], t, 0.0)
    z = np.ldexp(z, -e[..., None])
    mag = np.abs(z)
    grid = (F8 if fmt == FP8 else F4)[:127 if fmt == FP8 else 8]
    mid = (grid[1:] + grid[:-1]) / 2
    i = np.searchsorted(mid, mag, side="left")
    tie = (mag == mid[np.minimum(i, len(mid) - 1)]) & (i % 2 == 1)
    code = (i + tie) + (np.signbit(z) * (128 if fmt == FP8 else 8))
    scale = np.where(finite, e + 127, 255)
    return code.astype(np.uint8).reshape(x.shape), scale.astype(np.uint8)


def pack(codes, fmt):
    """One code per value -> the stored bytes."""
    return codes if fmt == FP8 else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(stored, fmt):
    if fmt == FP8:
        return stored
    return np.stack([stored & 15, stored >> 4], -1).reshape(*stored.shape[:-1], -1)


def values(codes, scales, fmt):
    """float64 values of codes (one per value) and scale bytes."""
    v = (F8 if fmt == FP8 else F4)[codes]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, -1)


def rows_of_cache(vc, vs):
    """V codes and scales as rows of keys: [b][Hkv][cap][dh/2] and [b][Hkv][cap][dh/32]."""
    b, h, g, q = vc.shape[:4]
    return (vc.transpose(0, 1, 2, 4, 3, 5).reshape(b, h, 8 * g, 2 * q),
            vs.transpose(0, 1, 2, 4, 3).reshape(b, h, 8 * g, -1))


def grouped(codes, scales):
    """The inverse of rows_of_cache."""
    b, h, cap, n = codes.shape
    vc = codes.reshape(b, h, cap // 8, 8, n // 2, 2).transpose(0, 1, 2, 4, 3, 5)
    vs = scales.reshape(b, h, cap // 8, 8, -1).transpose(0, 1, 2, 4, 3)
    return np.ascontiguousarray(vc), np.ascontiguousarray(vs)


def norm(h, delta, gain, eps):
    """(h + delta in float32, its RMS norm times gain in float64)."""
    h = h.astype(np.float32)
    if delta is not None:
        h = (h + delta.astype(np.float32)).astype(np.float32)
    y = h.astype(np.float64)
    with np.errstate(all="ignore"):
        return h, y * gain.astype(np.float64) / np.sqrt((y * y).mean(-1, keepdims=True) + eps)


def product_bound(x, w, scaled):
    """Largest error of the float32 product of x [M][K] and w [N][K].

    Sums in float32: K additions, each off by at most 2^-23 (the matrix
    instructions drop what lies below the last bit) of a partial sum that
    sum |x w| bounds.  The scaled instruction on top aligns the 8 products of
    consecutive k to the largest of them and keeps 13 bits below its leading
    one: each of the other 7 loses less than 2^-13 of it."""
    p = np.abs(x[:, None, :] * w[None, :, :])
    K = p.shape[-1]
    b = p.sum(-1) * K * 2.0 ** -23
    if scaled:
        b = b + 7 * 2.0 ** -13 * p.reshape(*p.shape[:2], -1, 8).max(-1).sum(-1)
    return b
