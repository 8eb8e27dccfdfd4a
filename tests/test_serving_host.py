"""Host-side refusals of the serving-step calls: every argument is checked before anything is enqueued (no GPU)."""
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


def _slots(lib, *, B=4, tok=16, page=8, n_pages=20, per=5, n_new=1 * MB, length=2 * MB, n_free=3 * MB, table=4 * MB,
           free=5 * MB, len_out=6 * MB, n_free_out=7 * MB, refused=8 * MB, first=9 * MB, start=10 * MB, seq=11 * MB,
           pos=12 * MB, slot=13 * MB):
    return lib.rm_page_slots(B, tok, page, n_pages, per, n_new, length, n_free, table, free, len_out, n_free_out, refused,
                             first, start, seq, pos, slot, None)


@pytest.mark.parametrize("kw,expected", [
    (dict(B=0), rm.RM_ERR_INVALID_ARG),
    (dict(B=(1 << 20) + 1), rm.RM_ERR_SHAPE),
    (dict(tok=0), rm.RM_ERR_INVALID_ARG),
    (dict(tok=1 << 30), rm.RM_ERR_SHAPE),
    (dict(page=0), rm.RM_ERR_INVALID_ARG),
    (dict(page=-4), rm.RM_ERR_INVALID_ARG),
    (dict(n_pages=0), rm.RM_ERR_INVALID_ARG),
    (dict(per=0), rm.RM_ERR_INVALID_ARG),
    (dict(n_pages=1 << 28, page=8), rm.RM_ERR_SHAPE),               # rows past int32
    (dict(n_pages=1 << 30, page=1), rm.RM_ERR_SHAPE),
    (dict(per=1 << 27), rm.RM_ERR_SHAPE),                           # 2^30 tokens
    (dict(n_new=None), rm.RM_ERR_INVALID_ARG),
    (dict(length=None), rm.RM_ERR_INVALID_ARG),
    (dict(n_free=None), rm.RM_ERR_INVALID_ARG),
    (dict(table=None), rm.RM_ERR_INVALID_ARG),
    (dict(start=None), rm.RM_ERR_INVALID_ARG),
    (dict(slot=None), rm.RM_ERR_INVALID_ARG),
    (dict(n_new=MB + 2), rm.RM_ERR_ALIGN),
    (dict(slot=13 * MB + 1), rm.RM_ERR_ALIGN),
    (dict(refused=8 * MB + 3), rm.RM_ERR_ALIGN),
    (dict(len_out=2 * MB + 4), rm.RM_ERR_INVALID_ARG),              # over len, not in its place
    (dict(len_out=1 * MB), rm.RM_ERR_INVALID_ARG),                  # over n_new
    (dict(n_free_out=2 * MB + 12), rm.RM_ERR_INVALID_ARG),          # the last length
    (dict(first=10 * MB - 16), rm.RM_ERR_INVALID_ARG),              # five entries: into start
    (dict(seq=12 * MB - 60), rm.RM_ERR_INVALID_ARG),                # into pos
    (dict(refused=4 * MB + 4 * 5 * 4 - 4), rm.RM_ERR_INVALID_ARG),  # the table's last entry
    (dict(free=4 * MB + 16), rm.RM_ERR_INVALID_ARG),
])
def test_page_slots_refuses(lib, kw, expected):
    assert _slots(lib, **kw) == expected
    assert rm.last_error() != ""


def _paged(lib, *, shape=(8, 2, 64, 1, 0.125, 0.0), N=3, seqs=3, page=16, n_pages=10, per=4, q=None, k=None, v=None,
           out=None, table=5 * MB, seq=None, pos=6 * MB, window=0, slopes=None, ws=64 * MB, ws_bytes=64 * MB):
    q, out = q or H(1 * MB, 0, 512, 64), out or H(4 * MB, 0, 512, 64)
    k, v = k or H(2 * MB, page * 128, 128, 64), v or H(3 * MB, page * 128, 128, 64)
    return lib.rm_paged_attention(ctypes.byref(rm.AttnShape(*shape)), N, seqs, page, n_pages, per, q, k, v, out, table, seq,
                                  pos, window, slopes, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,expected", [
    (dict(shape=(8, 3, 64, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 60, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 264, 1, 0.1, 0.0)), rm.RM_ERR_SHAPE),
    (dict(shape=(8, 2, 64, 2, 0.1, 0.0)), rm.RM_ERR_DTYPE),
    (dict(shape=(8, 2, 64, 1, 0.0, 0.0)), rm.RM_ERR_INVALID_ARG),
    (dict(shape=(8, 2, 64, 1, 0.1, -1.0)), rm.RM_ERR_INVALID_ARG),
    (dict(shape=(8, 2, 64, 1, 1e-10, 1e30)), rm.RM_ERR_INVALID_ARG),
    (dict(N=0), rm.RM_ERR_INVALID_ARG),
    (dict(seqs=0), rm.RM_ERR_INVALID_ARG),
    (dict(seqs=2), rm.RM_ERR_SHAPE),                                # no seq: a table for every token
    (dict(N=1 << 21, seqs=1 << 21), rm.RM_ERR_SHAPE),
    (dict(page=0), rm.RM_ERR_INVALID_ARG),
    (dict(n_pages=0), rm.RM_ERR_INVALID_ARG),
    (dict(per=0), rm.RM_ERR_INVALID_ARG),
    (dict(per=1 << 26), rm.RM_ERR_SHAPE),
    (dict(N=1 << 17, seqs=1 << 17, per=1 << 22), rm.RM_ERR_SHAPE),  # more tiles than a whole number counts
    (dict(n_pages=1 << 27), rm.RM_ERR_SHAPE),
    (dict(window=-1), rm.RM_ERR_INVALID_ARG),
    (dict(q=H(None, 0, 512, 64)), rm.RM_ERR_INVALID_ARG),
    (dict(k=H(None, 2048, 128, 64)), rm.RM_ERR_INVALID_ARG),
    (dict(q=H(MB + 8, 0, 512, 64)), rm.RM_ERR_ALIGN),
    (dict(k=H(2 * MB, 2048, 132, 64)), rm.RM_ERR_ALIGN),
    (dict(v=H(3 * MB, -2048, 128, 64)), rm.RM_ERR_SHAPE),
    (dict(v=H(3 * MB, 1 << 61, 128, 64)), rm.RM_ERR_SHAPE),
    (dict(out=H(4 * MB, 0, 512, 0)), rm.RM_ERR_SHAPE),              # heads on top of each other
    (dict(table=None), rm.RM_ERR_INVALID_ARG),
    (dict(pos=None), rm.RM_ERR_INVALID_ARG),
    (dict(table=5 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(pos=6 * MB + 1), rm.RM_ERR_ALIGN),
    (dict(seq=7 * MB + 3), rm.RM_ERR_ALIGN),
    (dict(slopes=7 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(out=H(1 * MB + 1024, 0, 512, 64)), rm.RM_ERR_INVALID_ARG),  # over q
    (dict(out=H(3 * MB, 0, 512, 64)), rm.RM_ERR_INVALID_ARG),       # over v
    (dict(table=4 * MB), rm.RM_ERR_INVALID_ARG),                    # out over the table
    (dict(pos=4 * MB + 64), rm.RM_ERR_INVALID_ARG),
    (dict(seq=4 * MB + 128), rm.RM_ERR_INVALID_ARG),
    (dict(slopes=4 * MB + 128), rm.RM_ERR_INVALID_ARG),
    (dict(ws=None), rm.RM_ERR_INVALID_ARG),
    (dict(ws=64 * MB + 128), rm.RM_ERR_ALIGN),
    (dict(ws_bytes=100), rm.RM_ERR_WORKSPACE),
    (dict(ws=4 * MB), rm.RM_ERR_INVALID_ARG),                       # over out
    (dict(ws=3 * MB - 256), rm.RM_ERR_INVALID_ARG),                 # over v
    (dict(ws=5 * MB - 256), rm.RM_ERR_INVALID_ARG),                 # over the table
])
def test_paged_attention_refuses(lib, kw, expected):
    assert _paged(lib, **kw) == expected
    assert rm.last_error() != ""


def test_paged_attention_workspace_refuses(lib):
    n = ctypes.c_size_t(0)
    s = ctypes.byref(rm.AttnShape(8, 2, 64, 1, 0.125, 0.0))
    assert lib.rm_paged_attention_workspace_size(s, 3, 16, 4, ctypes.byref(n)) == rm.RM_OK
    assert n.value % 256 == 0
    assert lib.rm_paged_attention_workspace_size(s, 1, 16, 8, ctypes.byref(n)) == rm.RM_OK and n.value == 0  # one wave's
    assert lib.rm_paged_attention_workspace_size(s, 3, 16, 4, None) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_paged_attention_workspace_size(None, 3, 16, 4, ctypes.byref(n)) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_paged_attention_workspace_size(s, 0, 16, 4, ctypes.byref(n)) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_paged_attention_workspace_size(s, 3, 0, 4, ctypes.byref(n)) == rm.RM_ERR_INVALID_ARG
    assert lib.rm_paged_attention_workspace_size(s, 3, 16, 1 << 27, ctypes.byref(n)) == rm.RM_ERR_SHAPE


def _norm(lib, *, B=2, T=3, d=64, xt=0, ft=1, ot=1, x=1 * MB, f=2 * MB, post=1, gain_post=3 * MB, gate=4 * MB, gate_s=64,
          xs=1.0, fs=1.0, y=5 * MB, gain_pre=6 * MB, scale=7 * MB, scale_s=64, shift=8 * MB, shift_s=64, eps=1e-6,
          out=9 * MB):
    return lib.rm_block_norm(B, T, d, xt, ft, ot, x, f, post, gain_post, gate, gate_s, xs, fs, y, gain_pre, scale, scale_s,
                             shift, shift_s, eps, out, None)


@pytest.mark.parametrize("kw,expected", [
    (dict(B=0), rm.RM_ERR_INVALID_ARG),
    (dict(T=0), rm.RM_ERR_INVALID_ARG),
    (dict(d=0), rm.RM_ERR_INVALID_ARG),
    (dict(d=60), rm.RM_ERR_SHAPE),
    (dict(d=32776), rm.RM_ERR_SHAPE),
    (dict(B=1 << 12, T=1 << 12), rm.RM_ERR_SHAPE),
    (dict(xt=2), rm.RM_ERR_DTYPE),
    (dict(ft=-1), rm.RM_ERR_DTYPE),
    (dict(ot=9), rm.RM_ERR_DTYPE),
    (dict(x=None), rm.RM_ERR_INVALID_ARG),
    (dict(f=None), rm.RM_ERR_INVALID_ARG),                          # with gate and norm_post
    (dict(f=None, post=0, gain_post=None), rm.RM_ERR_INVALID_ARG),  # with gate
    (dict(post=0), rm.RM_ERR_INVALID_ARG),                          # a gain without its norm
    (dict(y=None, out=None), rm.RM_ERR_INVALID_ARG),
    (dict(out=None), rm.RM_ERR_INVALID_ARG),                        # gain_pre without out
    (dict(out=None, gain_pre=None, scale=None), rm.RM_ERR_INVALID_ARG),
    (dict(eps=-1.0), rm.RM_ERR_INVALID_ARG),
    (dict(eps=float("nan")), rm.RM_ERR_INVALID_ARG),
    (dict(xs=float("inf")), rm.RM_ERR_INVALID_ARG),
    (dict(fs=float("nan")), rm.RM_ERR_INVALID_ARG),
    (dict(x=MB + 8), rm.RM_ERR_ALIGN),
    (dict(f=2 * MB + 2), rm.RM_ERR_ALIGN),
    (dict(gate=4 * MB + 4), rm.RM_ERR_ALIGN),
    (dict(gain_pre=6 * MB + 4), rm.RM_ERR_ALIGN),
    (dict(shift_s=66), rm.RM_ERR_ALIGN),
    (dict(gate_s=-64), rm.RM_ERR_SHAPE),
    (dict(scale_s=1 << 60), rm.RM_ERR_SHAPE),
    (dict(y=1 * MB + 256), rm.RM_ERR_INVALID_ARG),                  # over x, not in its place
    (dict(y=2 * MB), rm.RM_ERR_INVALID_ARG),                        # over f
    (dict(out=1 * MB), rm.RM_ERR_INVALID_ARG),                      # over x
    (dict(out=2 * MB, ot=0), rm.RM_ERR_INVALID_ARG),                # over f of another type
    (dict(out=2 * MB + 128), rm.RM_ERR_INVALID_ARG),                # over f, not in its place
    (dict(out=5 * MB), rm.RM_ERR_INVALID_ARG),                      # over y
    (dict(out=3 * MB), rm.RM_ERR_INVALID_ARG),                      # over a gain
    (dict(y=8 * MB), rm.RM_ERR_INVALID_ARG),                        # over the shift
    (dict(y=4 * MB + 64 * 4 * 8, gate_s=64 * 8), rm.RM_ERR_INVALID_ARG),  # over the last sample's gate
])
def test_block_norm_refuses(lib, kw, expected):
    assert _norm(lib, **kw) == expected
    assert rm.last_error() != ""


def test_the_binding_refuses_cpu_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(2, 4, 8)
    with pytest.raises(ValueError):
        rm.rm_page_slots(i, i, torch.zeros((4, 2), dtype=torch.int32), i, i[:1], torch.zeros(5, dtype=torch.int32), i, i, i,
                         i, 4)
    with pytest.raises(ValueError):
        rm.rm_paged_attention(x, x[None], x[None], torch.zeros((2, 1), dtype=torch.int32), i[:2], torch.zeros_like(x), None)
    with pytest.raises(ValueError):
        rm.rm_block_norm(x, x, None, torch.zeros_like(x))
