"""Host-side refusals of the attention-side calls: every argument is checked before anything is enqueued (no GPU)."""
import ctypes
import os

import pytest
import torch

import paper_2609_19104_amd as rm

MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rm.LIB_PATH):
        pytest.skip("librmuscle.so not built")
    return rm.load_library()


def H(at, batch, token, head):
    return ctypes.byref(rm.Heads(at, batch, token, head))


def _span(lib, *, shape=(8, 2, 64, 1, 0.125, 0.0), B=2, T=4, N=100, q=None, k=None, v=None, out=None, span=None, slopes=None,
          q_start=None, ws=None, ws_bytes=0):
    q = q or H(1 * MB, T * 512, 512, 64)
    k = k or H(2 * MB, N * 128, 128, 64)
    v = v or H(3 * MB, N * 128, 128, 64)
    out = out or H(4 * MB, T * 512, 512, 64)
    return lib.rm_span_attention(ctypes.byref(rm.AttnShape(*shape)), B, T, N, q, k, v, out, span, slopes, q_start, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,expected", [
    (dict(shape=(8, 3, 64, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(0, 0, 64, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 60, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 264, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 64, 5, 0.1, 0.0)), rm.RM_ERR_DTYPE),
    (dict(shape=(8, 2, 64, 1, float("nan"), 0.0)), rm.RM_ERR_INVALID_ARG),
    (dict(shape=(8, 2, 64, 1, float("inf"), 0.0)), rm.RM_ERR_INVALID_ARG),
    (dict(shape=(8, 2, 64, 1, 0.1, -1.0)), rm.RM_ERR_INVALID_ARG),
    (dict(shape=(8, 2, 64, 1, 0.1, float("inf"))), rm.RM_ERR_INVALID_ARG),
    (dict(B=0), rm.RM_ERR_INVALID_ARG),
    (dict(T=0), rm.RM_ERR_INVALID_ARG),
    (dict(N=-1), rm.RM_ERR_SHAPE),
    (dict(N=1 << 30), rm.RM_ERR_SHAPE),
    (dict(T=1 << 30), rm.RM_ERR_SHAPE),
    (dict(q=H(None, 2048, 512, 64)), rm.RM_ERR_INVALID_ARG),
    (dict(B=1 << 23, T=1), rm.RM_ERR_SHAPE),                        # more workgroups than a launch takes
    (dict(q=H(MB + 8, 2048, 512, 64)), rm.RM_ERR_ALIGN),
    (dict(k=H(2 * MB, 12800, 132, 64)), rm.RM_ERR_ALIGN),
    (dict(k=H(2 * MB, 12800, -128, 64)), rm.RM_ERR_SHAPE),
    (dict(k=H(2 * MB, 1 << 62, 128, 64)), rm.RM_ERR_SHAPE),
    (dict(v=H(2 * MB, 0, 8 * MB, 64)), rm.RM_ERR_SHAPE),            # 16 MiB from key to key
    (dict(out=H(4 * MB, 2048, 512, 0)), rm.RM_ERR_SHAPE),           # heads on top of each other
    (dict(out=H(4 * MB, 2048, 256, 64)), rm.RM_ERR_SHAPE),          # tokens into each other
    (dict(out=H(1 * MB + 1024, 2048, 512, 64)), rm.RM_ERR_INVALID_ARG),  # over q
    (dict(out=H(3 * MB, 2048, 512, 64)), rm.RM_ERR_INVALID_ARG),    # over v
    (dict(span=4 * MB), rm.RM_ERR_INVALID_ARG),                     # out over the spans
    (dict(span=5 * MB + 4), rm.RM_ERR_ALIGN),
    (dict(slopes=5 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(slopes=4 * MB), rm.RM_ERR_INVALID_ARG),
    (dict(slopes=5 * MB, q_start=4 * MB), rm.RM_ERR_INVALID_ARG),
    (dict(N=100000, k=H(64 * MB, 0, 128, 64), v=H(128 * MB, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),  # needs a workspace
    (dict(N=100000, k=H(64 * MB, 0, 128, 64), v=H(128 * MB, 0, 128, 64), ws=256 * MB, ws_bytes=100), rm.RM_ERR_WORKSPACE),
    (dict(N=100000, k=H(64 * MB, 0, 128, 64), v=H(128 * MB, 0, 128, 64), ws=256 * MB + 16, ws_bytes=1 << 30),
     rm.RM_ERR_ALIGN),
    (dict(N=100000, k=H(64 * MB, 0, 128, 64), v=H(128 * MB, 0, 128, 64), ws=4 * MB, ws_bytes=1 << 30),
     rm.RM_ERR_INVALID_ARG),                                        # workspace over out
    (dict(N=100000, k=H(64 * MB, 0, 128, 64), v=H(128 * MB, 0, 128, 64), ws=64 * MB, ws_bytes=1 << 30),
     rm.RM_ERR_INVALID_ARG),                                        # workspace over k
])
def test_span_attention_refuses(lib, kw, expected):
    assert _span(lib, **kw) == expected
    assert rm.last_error() != ""


def _prefix(lib, *, shape=(8, 2, 64, 1, 0.125, 0.0), G=2, per=3, T=4, P=100, S=20, q=None, kp=None, vp=None, plen=None,
            ko=None, vo=None, olen=None, out=None, ws=None, ws_bytes=0):
    q = q or H(1 * MB, T * 512, 512, 64)
    kp, vp = kp or H(2 * MB, P * 128, 128, 64), vp or H(3 * MB, P * 128, 128, 64)
    ko, vo = ko or H(5 * MB, S * 128, 128, 64), vo or H(6 * MB, S * 128, 128, 64)
    out = out or H(4 * MB, T * 512, 512, 64)
    return lib.rm_prefix_attention(ctypes.byref(rm.AttnShape(*shape)), G, per, T, P, S, q, kp, vp, plen, ko, vo, olen, 0, out, ws,
                                   ws_bytes, None)


@pytest.mark.parametrize("kw,expected", [
    (dict(shape=(8, 2, 64, 2, 0.1, 0.0)), rm.RM_ERR_DTYPE),
    (dict(G=0), rm.RM_ERR_INVALID_ARG),
    (dict(per=0), rm.RM_ERR_INVALID_ARG),
    (dict(P=-1), rm.RM_ERR_SHAPE),
    (dict(S=1 << 30), rm.RM_ERR_SHAPE),
    (dict(per=1 << 20, T=1 << 10), rm.RM_ERR_SHAPE),
    (dict(kp=H(None, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),
    (dict(vo=H(6 * MB + 4, 0, 128, 64)), rm.RM_ERR_ALIGN),
    (dict(plen=7 * MB + 1), rm.RM_ERR_ALIGN),
    (dict(olen=4 * MB), rm.RM_ERR_INVALID_ARG),                     # out over the lengths
    (dict(out=H(5 * MB, 2048, 512, 64)), rm.RM_ERR_INVALID_ARG),    # over the own keys
    (dict(P=100000, kp=H(64 * MB, 0, 128, 64), vp=H(128 * MB, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),  # no workspace
])
def test_prefix_attention_refuses(lib, kw, expected):
    assert _prefix(lib, **kw) == expected
    assert rm.last_error() != ""


def test_workspace_sizes(lib):
    n = ctypes.c_size_t(1)
    s = ctypes.byref(rm.AttnShape(8, 2, 64, 1, 0.125, 0.0))
    assert lib.rm_span_attention_workspace_size(s, 1, 16384, 4096, ctypes.byref(n)) == rm.RM_OK and n.value == 0
    assert lib.rm_span_attention_workspace_size(s, 1, 1, 65536, ctypes.byref(n)) == rm.RM_OK and n.value > 0
    assert n.value % 256 == 0
    assert lib.rm_span_attention_workspace_size(s, 1, 1, 65536, None) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_span_attention_workspace_size(None, 1, 1, 65536, ctypes.byref(n)) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_prefix_attention_workspace_size(s, 1, 1, 1, 65536, 0, ctypes.byref(n)) == rm.RM_OK and n.value > 0
    assert lib.rm_prefix_attention_workspace_size(s, 0, 1, 1, 65536, 0, ctypes.byref(n)) == rm.RM_ERR_INVALID_ARG


def _rope(lib, *, N=5, Hq=4, Hk=2, D=64, ind=1, outd=1, q=None, k=None, v=None, qo=None, ko=None, vo=None, rows=9,
          pos=7 * MB, slot=8 * MB, f=9 * MB, rot=64, gq=None, gk=None, eps=1e-6):
    q, k = q or H(1 * MB, 0, 256, 64), k or H(2 * MB, 0, 128, 64)
    v, qo = v or H(3 * MB, 0, 128, 64), qo or H(4 * MB, 0, 256, 64)
    ko, vo = ko or H(5 * MB, 0, 128, 64), vo or H(6 * MB, 0, 128, 64)
    return lib.rm_qk_norm_rope(N, Hq, Hk, D, ind, outd, q, k, v, qo, ko, vo, rows, pos, slot, f, rot, 0, gq, gk, eps,
                               None)


@pytest.mark.parametrize("kw,expected", [
    (dict(N=-1), rm.RM_ERR_INVALID_ARG),
    (dict(Hq=0), rm.RM_ERR_INVALID_ARG),
    (dict(rows=-1), rm.RM_ERR_INVALID_ARG),
    (dict(D=36), rm.RM_ERR_SHAPE),
    (dict(D=512, rot=0), rm.RM_ERR_SHAPE),
    (dict(rot=66), rm.RM_ERR_SHAPE),
    (dict(rot=68), rm.RM_ERR_SHAPE),
    (dict(rot=-4), rm.RM_ERR_SHAPE),
    (dict(ind=3), rm.RM_ERR_DTYPE),
    (dict(outd=-1), rm.RM_ERR_DTYPE),
    (dict(eps=-1.0), rm.RM_ERR_INVALID_ARG),
    (dict(eps=float("nan")), rm.RM_ERR_INVALID_ARG),
    (dict(slot=None, rows=4), rm.RM_ERR_SHAPE),
    (dict(N=1 << 29), rm.RM_ERR_SHAPE),
    (dict(N=1 << 26, rows=1 << 26), rm.RM_ERR_SHAPE),
    (dict(pos=None), rm.RM_ERR_INVALID_ARG),
    (dict(f=None), rm.RM_ERR_INVALID_ARG),
    (dict(pos=7 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(gk=7 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(q=H(MB + 2, 0, 256, 64)), rm.RM_ERR_ALIGN),
    (dict(q=H(MB, 0, 257, 64)), rm.RM_ERR_ALIGN),
    (dict(qo=H(1 * MB, 0, 256, 64)), rm.RM_ERR_INVALID_ARG),        # over q
    (dict(vo=H(5 * MB + 256, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),  # over k_out
    (dict(ko=H(7 * MB, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),        # over pos
    (dict(ko=H(5 * MB, 0, 64, 64)), rm.RM_ERR_SHAPE),               # rows into each other
    (dict(vo=H(None, 0, 128, 64)), rm.RM_ERR_INVALID_ARG),
])
def test_qk_norm_rope_refuses(lib, kw, expected):
    assert _rope(lib, **kw) == expected
    assert rm.last_error() != ""


@pytest.mark.parametrize("args,expected", [
    ((0, 4, 4, 1, 0, None, None, None, None, MB), rm.RM_ERR_INVALID_ARG),
    ((1, 0, 4, 1, 0, None, None, None, None, MB), rm.RM_ERR_INVALID_ARG),
    ((1, 4, 0, 1, 0, None, None, None, None, MB), rm.RM_ERR_INVALID_ARG),
    ((1, 4, 1 << 30, 1, 0, None, None, None, None, MB), rm.RM_ERR_SHAPE),
    ((1, 4, 4, 1, -1, None, None, None, None, MB), rm.RM_ERR_INVALID_ARG),
    ((1 << 24, 1, 4, 1, 0, None, None, None, None, MB), rm.RM_ERR_SHAPE),
    ((1, 4, 4, 0, 0, None, None, 2 * MB, None, MB), rm.RM_ERR_INVALID_ARG),  # prefix lengths without causal
    ((1, 4, 4, 1, 0, None, None, None, None, None), rm.RM_ERR_INVALID_ARG),
    ((1, 4, 4, 1, 0, None, None, None, None, MB + 4), rm.RM_ERR_ALIGN),
    ((1, 4, 4, 1, 0, 2 * MB + 1, None, None, None, MB), rm.RM_ERR_ALIGN),
    ((1, 4, 4, 1, 0, None, None, None, MB + 16, MB), rm.RM_ERR_INVALID_ARG),  # span over doc
])
def test_attn_spans_refuses(lib, args, expected):
    assert lib.rm_attn_spans(*args, None) == expected
    assert rm.last_error() != ""


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(1, 4, 2, 8)
    with pytest.raises(ValueError):
        rm.rm_span_attention(x, x, x, torch.zeros_like(x), None)
    with pytest.raises(ValueError):
        rm.rm_prefix_attention(x, x, x, x, x, torch.zeros_like(x), None)
    with pytest.raises(ValueError):
        rm.rm_qk_norm_rope(x[0], x[0], None, x[0], x[0], None, torch.zeros(4, dtype=torch.int32), None)
    with pytest.raises(ValueError):
        rm.rm_attn_spans(torch.zeros((1, 4, 2), dtype=torch.int32), 4)


@pytest.mark.parametrize("scale,cap,ok", [
    (0.125, 0.0, True), (0.125, 30.0, True), (0.125, 1e8, True), (0.125, 1e-30, True), (1.0, 1e37, True),
    (0.125, 3e38, False),   # the cap in powers of two is infinite
    (1e-10, 1e30, False),   # scale / softcap is denormal
    (1.0, 1e-39, False),    # or infinite
])
def test_softcaps_that_float32_does_not_hold(lib, scale, cap, ok):
    n = ctypes.c_size_t(1)
    for dtype in (rm.RM_BF16, rm.RM_F32):
        s = ctypes.byref(rm.AttnShape(8, 2, 64, dtype, scale, cap))
        want = rm.RM_OK if ok else rm.RM_ERR_INVALID_ARG
        assert lib.rm_span_attention_workspace_size(s, 1, 4, 64, ctypes.byref(n)) == want
        assert lib.rm_prefix_attention_workspace_size(s, 1, 1, 4, 64, 4, ctypes.byref(n)) == want
        if not ok:
            assert _span(lib, shape=(8, 2, 64, dtype, scale, cap), out=H(4 * MB, 4096, 1024, 128)) == want


@pytest.mark.parametrize("N,qo,ko,vo,ok", [
    # rows of one buffer, 4 + 2 + 2 heads of 128 bytes: q_out, k_out, v_out side by side
    (9, (0, 512, 64), (512, 512, 64), (768, 512, 64), True),
    (9, (0, 512, 64), (384, 512, 64), (768, 512, 64), False),          # the keys begin in the queries' last head
    (9, (0, 512, 64), (512, 512, 64), (640, 512, 64), False),          # the values in the keys' second head
    (9, (0, 512, 64), (512, 512, 64), (896, 512, 64), False),          # the values' second head in the next row's queries
    (9, (0, 512, 64), (512 + 1024, 512, 64), (768 + 2048, 512, 64), True),  # keys a row further, values two
    (9, (0, 512, 64), (512, 448, 64), (768, 512, 64), False),          # another step
    (1, (0, 512, 64), (512, 512, 64), (768, 512, 64), True),           # one token
    # caches beside the queries' own buffer: keys beside values in a row, in a head, and by heads
    (9, (8 * MB, 256, 64), (0, 256, 64), (256, 256, 64), True),
    (9, (8 * MB, 256, 64), (0, 256, 128), (128, 256, 128), True),
    (9, (8 * MB, 256, 64), (0, 64, 2 * 9 * 64), (9 * 128, 64, 2 * 9 * 64), True),
    (9, (8 * MB, 256, 64), (0, 64, 2 * 9 * 64), (8 * 128, 64, 2 * 9 * 64), False),
    (9, (8 * MB, 256, 64), (0, 256, 128), (0, 256, 128), False),       # the same
    (9, (8 * MB, 256, 64), (0, 256, 128), (64, 256, 128), False),      # half a vector into each other
    (9, (8 * MB, 256, 64), (256, 256, 128), (0, 256, 128), False),     # the same, a row apart
])
def test_outputs_in_one_buffer(lib, N, qo, ko, vo, ok):
    """Distinct elements are told from shared ones before the pointers meet the inputs: pos lies in q_out, so that no
    call reaches the GPU."""
    at = 64 * MB
    heads = [H(at + o, 0, t, h) for o, t, h in (qo, ko, vo)]
    status = _rope(lib, N=N, rows=9, qo=heads[0], ko=heads[1], vo=heads[2], slot=None, pos=at + qo[0])
    assert status == rm.RM_ERR_INVALID_ARG
    assert rm.last_error() == ("an output overlaps an input" if ok else "the outputs overlap each other")


def test_outputs_in_one_buffer_against_their_bytes(lib):
    """Random layouts: every one that is taken has no byte in two outputs."""
    import random

    r = random.Random(5)
    taken = 0
    for _ in range(3000):
        N, Hq, Hk, D = r.randint(1, 4), r.choice((2, 4)), r.choice((1, 2)), 8
        rows = N + r.randint(0, 2)
        def axes(n, h):  # noqa: E306
            t, s = r.choice([(8 * h * r.randint(1, 3), 8), (8, 8 * n * r.randint(1, 3)), (16 * h, 16), (64, 8), (64, 16)])
            return t, s
        steps = [axes(N, Hq), axes(rows, Hk)]
        steps.append(steps[1] if r.random() < 0.7 else axes(rows, Hk))
        if r.random() < 0.3:
            steps = [(64, 8)] * 3
        at = [16 * r.randint(0, 20) for _ in range(3)]
        def covered(at, t, s, n, h):  # noqa: E306
            return [at + (i * t + j * s) * 2 + c for i in range(n) for j in range(h) for c in range(2 * D)]
        cells = [covered(at[i], *steps[i], (N, rows, rows)[i], (Hq, Hk, Hk)[i]) for i in range(3)]
        if any(len(set(c)) != len(c) for c in cells):
            continue
        shared = len(set().union(*cells)) != sum(len(c) for c in cells)
        heads = [H(64 * MB + at[i], 0, *steps[i]) for i in range(3)]
        assert _rope(lib, N=N, Hq=Hq, Hk=Hk, D=D, rot=8, rows=rows, q=H(MB, 0, 64, 8), k=H(2 * MB, 0, 64, 8),
                     v=H(3 * MB, 0, 64, 8), qo=heads[0], ko=heads[1], vo=heads[2], slot=None,
                     pos=64 * MB + at[0]) != rm.RM_OK
        if rm.last_error() == "an output overlaps an input":
            assert not shared
            taken += 1
    assert taken > 300


def test_most_tokens(lib):
    """A wave a token and four waves a workgroup: below 2^24 workgroups, 2^32 threads.  The tokens that are taken get as
    far as the overlap of q_out with q, 1 MB behind it."""
    most = (1 << 26) - 4
    for n in (most, most + 1, most + 2, most + 3):
        want = rm.RM_ERR_INVALID_ARG if n <= most else rm.RM_ERR_SHAPE
        assert _rope(lib, N=n, rows=n, Hq=2, Hk=1, slot=None, qo=H(2 * MB, 0, 256, 64)) == want, n


@pytest.mark.parametrize("Hq,Hk,D,per,T,P,S,slices", [
    (8, 8, 128, 32, 1, 128, 256, 2),    # 8 workgroups with 32 samples' keys each
    (4, 1, 128, 16, 1, 256, 512, 2),    # 4 rows a sample, 8 samples a block
    (8, 8, 64, 32, 1, 0, 512, 2),       # own keys alone
    (8, 1, 256, 3, 51, 0, 8192, 2),     # blocks that hold the end of one sample and the begin of the next
    (8, 8, 128, 32, 1, 128, 0, 1),      # one tile
    (8, 8, 128, 1, 1, 128, 128, 1),
])
def test_slices_count_the_own_keys_of_every_sample_of_a_block(lib, Hq, Hk, D, per, T, P, S, slices):
    n = ctypes.c_size_t(0)
    s = ctypes.byref(rm.AttnShape(Hq, Hk, D, 1, 0.1, 0.0))
    assert lib.rm_prefix_attention_workspace_size(s, 1, per, T, P, S, ctypes.byref(n)) == rm.RM_OK
    one = per * T * Hq * (D * 4 + 8)
    assert n.value >= slices * one if slices > 1 else n.value == 0
