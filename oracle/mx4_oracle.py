"""CPU oracle of normalised, turned heads and of the 4-bit cache.  TEST INFRASTRUCTURE ONLY, float64, no code shared with the kernels.

    norm_rotary            rows over their root mean square, times the weight, then oracle.cache_oracle.rotary
    norm_rotary_gradient   the transpose of its derivative, row by row as a matrix: d(x / s) / dx = (I - u u' / D) / s with u = x / s
    hold                   rows of 32-channel blocks: scale by trial, each value by the distance to all sixteen codes
    pages_of / rows_of     the bytes of a page: codes [page][D / 2], even channel in the low half, then scales [D / 32][page]

Pins (tests/test_oracle_mx4_pins.py): differences, torch's own norm, values that the format holds exactly, ties, borders of the scale, round trips,
numbers that are not finite.
"""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle as co

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEAST, MOST = 1, 252                               # scale bytes


def _size(x, eps):
    return np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def norm_rotary(x, weight, positions, inv_freq, sections, *, eps, interleaved=False, norm=True):
    """x [B, heads, S, D] -> float64 of its shape.  weight [D] or None."""
    x = np.array(x, dtype=np.float64)
    z = x / _size(x, eps) if norm else x
    if weight is not None:
        z = z * np.asarray(weight, dtype=np.float64)
    return co.rotary(z, positions, inv_freq, sections, interleaved=interleaved)


def norm_rotary_gradient(x, weight, dy, positions, inv_freq, sections, *, eps, interleaved=False):
    """-> dx of x's shape, dw [D]; and for tolerances the sums of magnitudes that they are made of."""
    x = np.array(x, dtype=np.float64)
    D = x.shape[-1]
    w = np.ones(D) if weight is None else np.asarray(weight, dtype=np.float64)
    dz = co.rotary(np.asarray(dy, dtype=np.float64), positions, inv_freq, sections, interleaved=interleaved, inverse=True)
    s = _size(x, eps)
    u, g = x / s, dz * w
    dx = (g - u * np.sum(u * g, axis=-1, keepdims=True) / D) / s
    length = pair_lengths(np.asarray(dy, dtype=np.float64), sections, interleaved)     # a turned pair is off by a part of its length
    dx_size = (np.abs(w) * length + np.abs(u) * np.sum(np.abs(u * w) * length, axis=-1, keepdims=True) / D) / s
    axes = (0, 1, 2)
    return dx, np.sum(dz * u, axis=axes), dx_size, np.sum(np.abs(u) * length, axis=axes)


def pair_lengths(x, sections, interleaved):
    n = sum(sections)
    length = np.abs(x)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        length[..., a] = length[..., b] = np.hypot(x[..., a], x[..., b])
    return length


def hold(x):
    """Rows x [..., D] -> codes [..., D] (0 .. 15), scale bytes [..., D / 32], and how far the nearest border of another code or scale is, relative to the
    value there (a result nearer than its own error may round to either side)."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (-1, 32))
    size = np.where(np.isnan(b), 0.0, np.abs(b))
    most = size.max(-1)
    E = np.full(most.shape, LEAST)
    gap_scale = np.full(most.shape, np.inf)
    for e in range(LEAST, MOST):
        border = 7.0 * 2.0 ** (e - 127)
        E = np.where(most >= border, e + 1, E)
        with np.errstate(divide="ignore", invalid="ignore"):
            gap_scale = np.minimum(gap_scale, np.where(most > 0, np.abs(most - border) / np.where(most > 0, most, 1.0), np.inf))
    t = np.minimum(size / 2.0 ** (E - 127.0)[..., None], 100.0)
    off = np.abs(t[..., None] - VALUES)
    nearest = off.min(-1, keepdims=True)
    tied = off == nearest
    # of two codes as near as each other the even one
    code = np.where(tied.sum(-1) == 2, np.where(tied[..., 0::2].any(-1), 2 * np.argmax(tied[..., 0::2], -1), 0), np.argmax(tied, -1))
    borders = (VALUES[1:] + VALUES[:-1]) / 2
    with np.errstate(divide="ignore", invalid="ignore"):
        gap = np.min(np.abs(t[..., None] - borders), -1) / np.where(t > 0, t, 1.0)
    gap = np.minimum(gap, np.nan_to_num(gap_scale, nan=np.inf)[..., None])
    code = code + 8 * (np.signbit(b) & ~np.isnan(b))
    return code.reshape(x.shape).astype(np.uint8), E.astype(np.uint8), gap.reshape(x.shape)


def values(codes, scales):
    """codes [..., D], scale bytes [..., D / 32] -> float64 [..., D]."""
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes % 8]
    return (v.reshape(v.shape[:-1] + (-1, 32)) * 2.0 ** (scales.astype(np.float64) - 127.0)[..., None]).reshape(v.shape)


def pages_of(codes, scales):
    """codes [pages, Hkv, page, D], scales [pages, Hkv, page, D / 32] -> uint8 [pages, Hkv, page * (D / 2 + D / 32)]."""
    n, h, page, D = codes.shape
    out = np.zeros((n, h, page * (D // 2 + D // 32)), dtype=np.uint8)
    for t in range(page):
        for c in range(D // 2):
            out[:, :, t * (D // 2) + c] = codes[:, :, t, 2 * c] + 16 * codes[:, :, t, 2 * c + 1]
        for s in range(D // 32):
            out[:, :, page * (D // 2) + s * page + t] = scales[:, :, t, s]
    return out


def rows_of(cache, page, D):
    """uint8 [pages, Hkv, bytes] -> codes [pages, Hkv, page, D] and scales [pages, Hkv, page, D / 32]."""
    n, h, _ = cache.shape
    codes, scales = np.zeros((n, h, page, D), dtype=np.uint8), np.zeros((n, h, page, D // 32), dtype=np.uint8)
    for t in range(page):
        for c in range(D // 2):
            byte = cache[:, :, t * (D // 2) + c]
            codes[:, :, t, 2 * c], codes[:, :, t, 2 * c + 1] = byte & 15, byte >> 4
        for s in range(D // 32):
            scales[:, :, t, s] = cache[:, :, page * (D // 2) + s * page + t]
    return codes, scales


def dense(cache, page, D):
    """uint8 [pages, Hkv, bytes] -> the bf16 cache that it stands for, float64 [pages, page, Hkv, D] as oracle.decode_oracle takes it."""
    return values(*rows_of(cache, page, D)).transpose(0, 2, 1, 3)
