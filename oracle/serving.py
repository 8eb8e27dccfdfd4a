"""A serving step around the layers, from its definitions: pages and slots request by request, attention over pages one key
at a time, block norms in float64.  Each of the computed values comes with what its callers need for an error bound."""
from __future__ import annotations

from typing import List, NamedTuple, Optional

import numpy as np

from .attention import attend


class Slots(NamedTuple):
    seq: List[int]
    pos: List[int]
    slot: List[int]
    first: List[int]
    start: List[int]
    length: List[int]
    n_free: int
    refused: int
    table: List[List[int]]
    free_pages: List[int]


def page_slots(n_new, length, table, free_pages, n_free: int, page: int, max_tok: int) -> Slots:
    per, n_pages = len(table[0]), len(free_pages)
    table, free_pages = [list(map(int, t)) for t in table], list(map(int, free_pages))
    length = [min(max(int(x), 0), per * page) for x in length]
    top = min(max(int(n_free), 0), n_pages)
    count = lambda tokens: -(-tokens // page)  # noqa: E731
    for b, n in enumerate(n_new):
        if n < 0:
            for i in range(count(length[b])):
                if top < n_pages:
                    free_pages[top] = table[b][i]
                top += 1
    top = min(top, n_pages)
    seq, pos, slot = [-1] * max_tok, [-1] * max_tok, [-1] * max_tok
    first, start, refused, wanted, taken = [0], [], 0, 0, 0
    for b, n in enumerate(int(x) for x in n_new):
        begin = first[-1]
        first.append(min(begin + max(n, 0), 1 << 30))
        if n < 0:
            length[b] = 0
            start.append(-1)
            continue
        want, old = 0, length[b]
        ok = old + n <= per * page and (n == 0 or first[-1] <= max_tok)
        if ok:
            want = count(old + n) - count(old)
            wanted += want
            ok = want == 0 or wanted <= top
        if ok:
            for i in range(want):
                table[b][count(old) + i] = free_pages[top - 1 - taken]
                taken += 1
            length[b] = old + n
        else:
            refused += 1
        start.append(old if ok else -1)
        for t in range(begin, min(first[-1], max_tok)):
            seq[t] = b
            if ok:
                p = pos[t] = old + t - begin
                pg = table[b][p // page]
                slot[t] = pg * page + p % page if 0 <= pg < n_pages else -1
    return Slots(seq, pos, slot, first, start, length, top - taken, refused, table, free_pages)


def paged_attention(q, k_cache, v_cache, table, seq, pos, window: int, scale: float, cap: float = 0.0, slopes=None,
                    heads: Optional[List[int]] = None):
    """q [N][Hq][D], caches [n_pages][page][Hk][D] -> (out, mag, big) as attend; heads: the query heads to compute."""
    N, Hq, D = q.shape
    n_pages, page, Hk = k_cache.shape[:3]
    seqs, per = table.shape
    out, mag, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros((N, Hq))
    for n in range(N):
        s, p = (n if seq is None else int(seq[n])), int(pos[n])
        if not 0 <= s < seqs or p < 0:
            continue
        j = np.arange(max(0, p - window + 1) if window else 0, min(p + 1, per * page), dtype=np.int64)
        pg = np.asarray(table[s], np.int64)[j // page]
        ok = (pg >= 0) & (pg < n_pages)
        j, pg = j[ok], pg[ok]
        if len(j) == 0:
            continue
        for h in range(Hq) if heads is None else heads:
            bias = None if slopes is None else -float(slopes[h]) * (p - j)[None].astype(np.float64)
            kv = h // (Hq // Hk)
            o, m, g = attend(q[n, h:h + 1], k_cache[pg, j % page, kv], v_cache[pg, j % page, kv],
                             np.ones((1, len(j)), bool), scale, cap, bias)
            out[n, h], mag[n, h], big[n, h] = o[0], m[0], g[0]
    return out, mag, big


class Norm(NamedTuple):
    y: np.ndarray
    out: np.ndarray
    mag: np.ndarray      # |x_scale x| + |f_scale gate norm_post(f)|: what roundings of u are relative to
    factor: np.ndarray   # d out / d u at a fixed norm: gain_pre (1 + scale) / sqrt(mean(u^2) + eps)


def block_norm(x, f, norm_post: bool, gain_post=None, gate=None, gain_pre=None, scale=None, shift=None,
               x_scale: float = 1.0, f_scale: float = 1.0, eps: float = 1e-6) -> Norm:
    """x, f [B][T][d]; gains [d]; gate, scale, shift [B][d]."""
    rms = lambda a: np.sqrt((a * a).mean(-1, keepdims=True) + eps)  # noqa: E731
    xs = x_scale * np.asarray(x, np.float64)
    term = np.zeros_like(xs)
    if f is not None:
        term = np.asarray(f, np.float64)
        if norm_post:
            term = term / rms(term)
        if gain_post is not None:
            term = term * gain_post
        if gate is not None:
            term = term * np.asarray(gate)[:, None]
        term = f_scale * term
    u = xs + term
    factor = np.ones_like(u) / rms(u)
    if gain_pre is not None:
        factor = factor * gain_pre
    if scale is not None:
        factor = factor * (1.0 + np.asarray(scale)[:, None])
    out = u * factor
    if shift is not None:
        out = out + np.asarray(shift)[:, None]
    return Norm(u, out, np.abs(xs) + np.abs(term), factor)
