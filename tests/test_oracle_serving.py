"""Pins of the serving-step oracle: hand-worked steps, invariants of the page tables, and special cases of the attention
and of the norm that other definitions give."""
import numpy as np
import pytest

from oracle import attention as att
from oracle import rms_norm, serving


def test_a_step_by_hand():
    # Pages of 4 tokens.  Request 0 goes on inside its page, 1 takes a page, 2 ends (two pages), 3 wants two pages.
    table = [[7, -1, -1], [3, -1, -1], [5, 2, -1], [-1, -1, -1]]
    s = serving.page_slots([1, 1, -1, 5], [2, 4, 6, 0], table, [6, 1, 9, 9, 9, 9, 9, 9, 9, 9], 2, 4, 8)
    assert s.free_pages[:4] == [6, 1, 5, 2]
    assert s.table == [[7, -1, -1], [3, 2, -1], [5, 2, -1], [5, 1, -1]]
    assert s.first == [0, 1, 2, 2, 7] and s.start == [2, 4, -1, 0]
    assert s.length == [3, 5, 0, 5] and s.n_free == 1 and s.refused == 0
    assert s.seq == [0, 1, 3, 3, 3, 3, 3, -1] and s.pos == [2, 4, 0, 1, 2, 3, 4, -1]
    assert s.slot == [30, 8, 20, 21, 22, 23, 4, -1]


def test_refusals_by_hand():
    # One free page: the first that wants it gets it, the next wants are refused, tokens that need no page are served.
    table = [[-1, -1], [-1, -1], [4, -1], [5, 6]]
    s = serving.page_slots([2, 1, 1, 3], [0, 0, 1, 3], table, [9, 0, 0, 0, 0, 0, 0, 0, 0, 0], 1, 2, 6)
    assert s.start == [0, -1, 1, -1]  # request 3: 6 tokens do not fit into 2 pages of 2
    assert s.refused == 2 and s.length == [2, 0, 2, 3] and s.n_free == 0
    assert s.slot == [18, 19, -1, 9, -1, -1] and s.seq == [0, 0, 1, 2, 3, 3]


@pytest.mark.parametrize("seed", range(6))
def test_no_page_has_two_owners(seed):
    rng = np.random.default_rng(seed)
    B, per, page, n_pages = 9, 6, int(rng.integers(1, 6)), 30
    length, table = [0] * B, [[-1] * per for _ in range(B)]
    free, n_free = list(rng.permutation(n_pages)), n_pages
    for _ in range(40):
        n_new = [-1 if rng.random() < 0.15 else int(rng.integers(0, 2 * page + 2)) for _ in range(B)]
        s = serving.page_slots(n_new, length, table, free, n_free, page, B * (2 * page + 2))
        length, table, free, n_free = s.length, s.table, s.free_pages, s.n_free
        held = [t[i] for b, t in enumerate(table) for i in range(-(-length[b] // page))]
        assert sorted(held + free[:n_free]) == list(range(n_pages))
        rows = [x for x in s.slot if x >= 0]
        assert len(set(rows)) == len(rows) and len(rows) == sum(x >= 0 for x in s.pos)


def test_paged_attention_is_span_attention_on_gathered_rows():
    rng = np.random.default_rng(3)
    N, Hq, Hk, D, page, per, n_pages = 3, 4, 2, 8, 5, 4, 13
    q, k, v = rng.normal(size=(N, Hq, D)), rng.normal(size=(n_pages, page, Hk, D)), rng.normal(size=(n_pages, page, Hk, D))
    table = rng.permutation(n_pages)[:N * per].reshape(N, per)
    pos, seq, slopes = np.array([0, 19, 11]), np.array([2, 0, 1]), np.array([0.3, 0.0, 0.1, 0.2])
    for window in (0, 1, 7):
        out = serving.paged_attention(q, k, v, table, seq, pos, window, 0.3, 5.0, slopes)[0]
        span = np.array([[[max(0, p - window + 1) if window else 0, p + 1]] for p in pos])
        kk, vv = (c[table[seq]].reshape(N, per * page, Hk, D) for c in (k, v))
        ref = att.span_attention(q[:, None], kk, vv, span, 0.3, 5.0, slopes, pos)[0][:, 0]
        np.testing.assert_allclose(out, ref, rtol=1e-12)
    k[table[seq[0], 0], 1:] = v[table[seq[0], 0], 1:] = np.nan  # behind the first token's position
    assert np.isfinite(serving.paged_attention(q, k, v, table, seq, pos, 0, 0.3)[0][0]).all()
    table[0, 0] = n_pages  # a page that is none: its keys are not there
    out = serving.paged_attention(q, k, v, table, None, np.array([4, -1, 3]), 0, 0.3)[0]
    assert (out[:2] == 0).all() and (out[2] != 0).all()


def test_block_norm_special_cases():
    rng = np.random.default_rng(4)
    x, f = rng.normal(size=(2, 3, 16)), rng.normal(size=(2, 3, 16))
    g, gate, scale, shift = rng.normal(size=16), rng.normal(size=(2, 16)), rng.normal(size=(2, 16)), rng.normal(size=(2, 16))
    r = serving.block_norm(x, None, False, gain_pre=g)
    np.testing.assert_allclose(r.y, x)
    np.testing.assert_allclose(r.out, rms_norm(x, g), rtol=1e-12)
    r = serving.block_norm(x, f, False, gate=gate, x_scale=0.5, f_scale=2.0)
    np.testing.assert_allclose(r.y[1, 2], 0.5 * x[1, 2] + 2 * gate[1] * f[1, 2])
    r = serving.block_norm(x, f, True, gain_post=g, scale=scale, shift=shift)
    np.testing.assert_allclose(r.y, x + rms_norm(f, g), rtol=1e-12)
    np.testing.assert_allclose(r.out[0, 1], rms_norm(r.y[0, 1], np.ones(16)) * (1 + scale[0]) + shift[0], rtol=1e-12)
