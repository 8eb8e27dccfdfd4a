"""Attention side of a layer in float64: head norms and rotations, key intervals, attention over intervals and over a
shared prefix.  Plain loops over heads and rows' definitions; keys that a row does not see are left out of its sums
altogether, so whatever they hold cannot reach it.

Each attention also returns what its callers need for an error bound: the same average over |v| and the largest
scale * sum |q_c| |k_c| among the seen keys."""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np


def norm_rope(x: np.ndarray, gain: Optional[np.ndarray], pos: np.ndarray, inv_freq: np.ndarray, eps: float,
              pairs: bool) -> np.ndarray:
    """x [N][H][D] -> normalized (gain not None) and rotated heads."""
    y = np.asarray(x, np.float64).copy()
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    half = len(inv_freq)
    ang = np.asarray(pos, np.float64)[:, None] * np.asarray(inv_freq, np.float64)[None, :]
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    i, j = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if pairs else (np.arange(half), np.arange(half) + half)
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i] = a * c - b * s
    y[..., j] = b * c + a * s
    return y


def spans(B: int, T: int, N: int, causal: bool, window: int, q_start=None, kv_len=None, prefix_len=None,
          doc=None) -> np.ndarray:
    """The definition of rm_attn_spans, row by row."""
    out = np.zeros((B, T, 2), np.int32)
    for b in range(B):
        kv = N if kv_len is None else min(max(int(kv_len[b]), 0), N)
        for i in range(T):
            p = (0 if q_start is None else int(q_start[b])) + i
            lo, hi = 0, kv
            if causal:
                hi = min(kv, max(p + 1, 0 if prefix_len is None else int(prefix_len[b])))
            if window > 0:
                lo = max(0, p - window + 1)
            if (causal or doc is not None) and not 0 <= p < kv:
                continue
            if doc is not None:
                if doc[b][p] < 0:
                    continue
                x = p
                while x > 0 and doc[b][x - 1] == doc[b][p]:
                    x -= 1
                y = p + 1
                while y < N and doc[b][y] == doc[b][p]:
                    y += 1
                lo, hi = max(lo, x), min(hi, y)
            if lo < hi:
                out[b, i] = lo, hi
    return out


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, seen: np.ndarray, scale: float, cap: float,
           bias: Optional[np.ndarray]) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """One head: q [T][D], k, v [N][D], seen bool [T][N], bias [T][N] added to the capped scores ->
    (out [T][D], the average of |v| [T][D], largest scale * sum |q||k| of the seen keys [T])."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    out, mag, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[0])
    for t in range(q.shape[0]):
        j = np.flatnonzero(seen[t])
        if len(j) == 0:
            continue
        s = scale * (k[j] @ q[t])
        big[t] = np.max(abs(scale) * (np.abs(k[j]) @ np.abs(q[t])))
        if cap:
            s = cap * np.tanh(s / cap)
        if bias is not None:
            s = s + bias[t, j]
        w = np.exp(s - np.max(s))
        w /= w.sum()
        out[t] = w @ v[j]
        mag[t] = w @ np.abs(v[j])
    return out, mag, big


def span_attention(q, k, v, span, scale: float, cap: float = 0.0, slopes=None, q_start=None):
    """q [B][T][Hq][D], k, v [B][N][Hk][D], span [B][T][2] -> (out, mag, big) as attend, for all heads."""
    B, T, Hq, D = q.shape
    N, Hk = k.shape[1], k.shape[2]
    out, mag, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, T, Hq))
    j = np.arange(N)
    for b in range(B):
        seen = (j >= span[b, :, :1]) & (j < span[b, :, 1:])
        at = np.arange(T) + (0 if q_start is None else int(q_start[b]))
        for h in range(Hq):
            bias = None if slopes is None else -float(slopes[h]) * np.abs(at[:, None] - j[None, :])
            kv = h // (Hq // Hk)
            out[b, :, h], mag[b, :, h], big[b, :, h] = attend(q[b, :, h], k[b, :, kv], v[b, :, kv], seen, scale, cap, bias)
    return out, mag, big


def prefix_attention(q, k_prefix, v_prefix, k_own, v_own, scale: float, cap: float = 0.0, prefix_len=None, own_len=None,
                     causal: bool = False):
    """q [B][T][Hq][D], prefix [G][P][Hk][D], own [B][S][Hk][D] -> (out, mag, big)."""
    B, T, Hq, D = q.shape
    G, P, Hk = k_prefix.shape[:3]
    S = k_own.shape[1]
    out, mag, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, T, Hq))
    for b in range(B):
        g = b // (B // G)
        p = P if prefix_len is None else min(max(int(prefix_len[g]), 0), P)
        n = S if own_len is None else min(max(int(own_len[b]), 0), S)
        j = np.arange(n)
        own = np.ones((T, n), bool)
        if causal:
            own = j[None, :] <= (n - T + np.arange(T))[:, None]
        seen = np.concatenate((np.ones((T, p), bool), own), 1)
        k = np.concatenate((k_prefix[g, :p], k_own[b, :n]))
        v = np.concatenate((v_prefix[g, :p], v_own[b, :n]))
        for h in range(Hq):
            kv = h // (Hq // Hk)
            out[b, :, h], mag[b, :, h], big[b, :, h] = attend(q[b, :, h], k[:, kv], v[:, kv], seen, scale, cap, None)
    return out, mag, big
