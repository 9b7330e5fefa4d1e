"""CPU oracle of the operators around a bounded key/value cache.  TEST INFRASTRUCTURE ONLY, float64, no code shared with the kernels.

    rotary        channel pairs as complex numbers times exp(i * position * frequency), pair by pair
    key_weights   full score matrix of the newest rows of one sequence, masked softmax, column sums over rows and the heads of a kv head
    evict         Python's sort on (protected, weight, slot)

Pins (tests/test_oracle_cache_pins.py): a turn by nothing and by a quarter, relative phase (the score of two turned rows depends on the
difference of their positions alone), the transpose as the inverse, weights that add up to the visible rows, the decode oracle's
probabilities, brute-force selections.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np


def rotary(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, sections: Sequence[int], *, interleaved: bool = False,
           inverse: bool = False) -> np.ndarray:
    """x [B, heads, S, D], positions [B, S, axes], inv_freq [pairs] -> float64 of x's shape."""
    y = np.array(x, dtype=np.float64)
    n = len(inv_freq)
    pair = 0
    for axis, count in enumerate(sections):
        for _ in range(count):
            a, b = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + n)
            t = positions[:, :, axis].astype(np.float64) * float(inv_freq[pair])
            z = (y[..., a] + 1j * y[..., b]) * np.exp((-1j if inverse else 1j) * t)[:, None, :]
            y[..., a], y[..., b] = z.real, z.imag
            pair += 1
    assert pair == n
    return y


def probabilities(q: np.ndarray, k: np.ndarray, length: int, *, scale: float, window: Optional[int] = None,
                  softcap: Optional[float] = None, slope: Optional[float] = None) -> np.ndarray:
    """One head: the T newest rows q [T, D] over the cached keys k [length, D] -> P [T, length] (rows without a key: zeros)."""
    T = q.shape[0]
    s = scale * (q.astype(np.float64) @ k.astype(np.float64).T)
    if softcap is not None:
        s = softcap * np.tanh(s / softcap)
    i, j = np.arange(length - T, length)[:, None], np.arange(length)[None, :]
    if slope is not None:
        s = s - slope * (i - j)
    seen = j <= i
    if window is not None:
        seen &= i - j <= window
    p = np.zeros((T, length))
    for r in range(T):
        if seen[r].any():
            e = np.where(seen[r], np.exp(np.where(seen[r], s[r], 0.0) - s[r][seen[r]].max()), 0.0)
            p[r] = e / e.sum()
    return p


def key_weights(q: np.ndarray, keys: Sequence[np.ndarray], weights: np.ndarray, *, scale: float, window: Optional[int] = None,
                softcap: Optional[float] = None, slopes: Optional[np.ndarray] = None) -> np.ndarray:
    """q [B, H, T, D], keys[b] [len_b, Hkv, D], weights [B, Hkv, C] -> the updated weights (float64)."""
    w = np.array(weights, dtype=np.float64)
    H, T, Hkv = q.shape[1], q.shape[2], w.shape[1]
    for b, k in enumerate(keys):
        n = k.shape[0]
        w[b, :, max(0, n - T):n] = 0.0
        for h in range(H):
            p = probabilities(q[b, h], k[:, h // (H // Hkv)], n, scale=scale, window=window, softcap=softcap,
                              slope=None if slopes is None else float(slopes[h]))
            w[b, h // (H // Hkv), :n] += p.sum(0)
    return w


def evict(weights: np.ndarray, lens: Sequence[int], budget: int, sinks: int, recent: int):
    """weights [B, Hkv, C] -> new lengths [B], kept slots [B, Hkv, budget] (-1 behind them)."""
    B, Hkv = weights.shape[:2]
    kept = np.full((B, Hkv, budget), -1, dtype=np.int32)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            def rank(j):
                w = float(weights[b, h, j])
                protected = j < sinks or j >= n - recent
                return (0 if protected else 1, 1 if w != w else 0, 0.0 if w != w else -w, j)
            stay = sorted(sorted(range(n), key=rank)[:min(n, budget)])
            kept[b, h, :len(stay)] = stay
    return np.minimum(np.asarray(lens), budget).astype(np.int32), kept
