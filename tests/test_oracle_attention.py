"""Pins of the attention oracle (float64): closed forms, torch's float64 operations, invariants."""
import numpy as np
import pytest
import torch

from oracle import attention as att


def _rng(*path):
    return np.random.default_rng([2609, 19104, 7, *path])


def test_one_key_gives_its_value_and_no_key_gives_zero():
    r = _rng(0)
    q, k, v = r.normal(size=(2, 3, 4, 8)), r.normal(size=(2, 5, 2, 8)), r.normal(size=(2, 5, 2, 8))
    span = np.zeros((2, 3, 2), np.int32)
    span[:, 0] = 2, 3
    o, mag, _ = att.span_attention(q, k, v, span, 0.3)
    for h in range(4):
        assert np.allclose(o[:, 0, h], v[:, 2, h // 2]) and np.allclose(mag[:, 0, h], np.abs(v[:, 2, h // 2]))
    assert not o[:, 1:].any()


def test_equal_scores_average_the_values():
    v = _rng(1).normal(size=(1, 6, 1, 8))
    o, _, _ = att.span_attention(np.zeros((1, 1, 1, 8)), np.ones((1, 6, 1, 8)), v, np.array([[[1, 5]]]), 1.0)
    assert np.allclose(o[0, 0, 0], v[0, 1:5, 0].mean(0))


@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_against_torch_float64(cap):
    r = _rng(2)
    B, T, N, Hq, Hk, D = 2, 5, 7, 4, 2, 8
    q, k, v = r.normal(size=(B, T, Hq, D)), r.normal(size=(B, N, Hk, D)), r.normal(size=(B, N, Hk, D))
    slopes = np.array([0.5, 0.25, 0.125, 0.0])
    span = att.spans(B, T, N, True, 0, q_start=[2, 2])
    o, _, _ = att.span_attention(q, k, v, span, 0.7, cap, slopes, [2, 2])
    tq, tk, tv = (torch.from_numpy(a) for a in (q, k, v))
    tk, tv = tk.repeat_interleave(2, 2), tv.repeat_interleave(2, 2)
    s = torch.einsum("bthd,bnhd->bhtn", tq, tk) * 0.7
    if cap:
        s = cap * torch.tanh(s / cap)
    dist = (torch.arange(T)[:, None] + 2 - torch.arange(N)).abs()
    s = s - torch.from_numpy(slopes)[None, :, None, None] * dist
    s = s.masked_fill(torch.arange(N) > torch.arange(T)[:, None] + 2, float("-inf"))
    ref = torch.einsum("bhtn,bnhd->bthd", torch.softmax(s, -1), tv)
    assert np.allclose(o, ref.numpy(), atol=1e-13)


def test_prefix_attention_is_span_attention_of_the_joined_keys():
    r = _rng(3)
    G, n, T, P, S, Hq, Hk, D = 2, 3, 2, 5, 4, 2, 1, 8
    q = r.normal(size=(G * n, T, Hq, D))
    kp, vp = r.normal(size=(2, G, P, Hk, D))
    ko, vo = r.normal(size=(2, G * n, S, Hk, D))
    pl, ol = [3, 5], [4, 0, 2, 1, 3, 4]
    o, _, _ = att.prefix_attention(q, kp, vp, ko, vo, 0.4, 0.0, pl, ol, True)
    for b in range(G * n):
        p, m = pl[b // n], ol[b]
        k = np.concatenate((kp[b // n, :p], ko[b, :m]))[None]
        v = np.concatenate((vp[b // n, :p], vo[b, :m]))[None]
        span = np.array([[[0, p + max(0, m - T + t + 1)] for t in range(T)]])
        ref, _, _ = att.span_attention(q[b:b + 1], k, v, span, 0.4)
        assert np.allclose(o[b:b + 1], ref, atol=1e-13)


def test_spans_hand_examples():
    assert att.spans(1, 4, 4, True, 0)[0].tolist() == [[0, 1], [0, 2], [0, 3], [0, 4]]
    assert att.spans(1, 4, 4, True, 2)[0].tolist() == [[0, 1], [0, 2], [1, 3], [2, 4]]
    assert att.spans(1, 4, 4, True, 0, prefix_len=[3])[0].tolist() == [[0, 3], [0, 3], [0, 3], [0, 4]]
    assert att.spans(1, 4, 4, False, 0, kv_len=[2])[0].tolist() == [[0, 2]] * 4
    assert att.spans(1, 4, 4, True, 0, kv_len=[2])[0].tolist() == [[0, 1], [0, 2], [0, 0], [0, 0]]
    assert att.spans(1, 5, 5, True, 0, doc=[[3, 3, -1, 3, 3]])[0].tolist() == [[0, 1], [0, 2], [0, 0], [3, 4], [3, 5]]
    assert att.spans(1, 5, 5, False, 0, doc=[[1, 1, 2, 2, 1]])[0].tolist() == [[0, 2], [0, 2], [2, 4], [2, 4], [4, 5]]
    assert att.spans(1, 2, 9, True, 0, q_start=[7])[0].tolist() == [[0, 8], [0, 9]]
    assert att.spans(1, 2, 9, True, 0, q_start=[-1])[0].tolist() == [[0, 0], [0, 1]]


def test_rotation_keeps_norms_and_depends_on_distances_only():
    r = _rng(4)
    x, y = r.normal(size=(2, 1, 1, 16))
    f = 10.0 ** -np.arange(8)
    rot = lambda a, p, pairs: att.norm_rope(a, None, np.array([p]), f, 0.0, pairs)  # noqa: E731
    for pairs in (False, True):
        assert np.allclose(np.linalg.norm(rot(x, 12345, pairs)), np.linalg.norm(x))
        assert np.allclose((rot(x, 9, pairs) * rot(y, 4, pairs)).sum(), (rot(x, 105, pairs) * rot(y, 100, pairs)).sum())
        assert np.array_equal(rot(x, 0, pairs), x)
    z = att.norm_rope(np.array([[[1.0, 0.0, 3.0, 4.0]]]), None, np.array([1]), np.array([np.pi / 2]), 0.0, False)
    assert np.allclose(z, [[[0.0, 1.0, 3.0, 4.0]]], atol=1e-15)


def test_norm_matches_torch():
    x = _rng(5).normal(size=(3, 2, 16))
    g = _rng(6).normal(size=16)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x), (16,), torch.from_numpy(g), 1e-6)
    assert np.allclose(att.norm_rope(x, g, np.zeros(3), np.zeros(0), 1e-6, False), ref.numpy(), atol=1e-14)
