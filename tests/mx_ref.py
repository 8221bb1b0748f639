"""Plain 64-bit implementation of the microscaled operators (numpy, from the
definitions in include/mpq.h), for the parity tests."""
from __future__ import annotations

import numpy as np

BLOCK, ROW = 32, 128
EMAX = {"fp4": 2, "fp8": 8}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # unit roundoff


def elements(fmt):
    """The values of the non-negative codes, ascending (fp8 without 0x7f)."""
    if fmt == "fp4":
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


def padded(x, to):
    return np.concatenate([x, np.zeros(x.shape[:-1] + (-x.shape[-1] % to,))], -1)


def quantize(x, fmt):
    """x [..., d] fp64, d a multiple of 32 -> codes [..., d] (one an element,
    sign at the top bit) and scale bytes [..., d / 32]."""
    vals = elements(fmt)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    a = np.abs(b).max(-1)
    e = np.frexp(np.where(a > 0, a, 1.0))[1] - 1
    s = np.maximum(np.where(a > 0, e + 127 - EMAX[fmt], 0), 0)
    y = np.minimum(np.abs(b) / np.ldexp(1.0, s - 127)[..., None], vals[-1])
    hi = np.clip(np.searchsorted(vals, y), 0, len(vals) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = y - vals[lo], vals[hi] - y
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = c | np.where(np.signbit(b), 8 if fmt == "fp4" else 128, 0)
    c = np.where(bad[..., None], 0, c)
    return c.reshape(x.shape).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def values(codes, scales, fmt):
    """[..., d] codes, [..., d / 32] scale bytes -> fp64 values."""
    vals = elements(fmt)
    top = 8 if fmt == "fp4" else 128
    mag = codes & (top - 1)
    v = np.where(mag < len(vals), vals[np.minimum(mag, len(vals) - 1)], np.nan)
    v = np.where(codes & top, -v, v)
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(f, BLOCK, -1)


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(bytes_):
    return np.stack([bytes_ & 15, bytes_ >> 4], -1).reshape(*bytes_.shape[:-1], -1)


def attend(q, k, v, scale):
    """One query head: q [D], k, v [n, D] fp64 -> o [D], lse, and the
    magnitude sum_j p_j |v_j| / sum_j p_j that errors scale with."""
    if len(k) == 0:
        return np.zeros(len(q)), -np.inf, np.zeros(len(q))
    s = k @ q * scale
    m = s.max()
    p = np.exp(s - m)
    return p @ v / p.sum(), m + np.log(p.sum()), p @ np.abs(v) / p.sum()
