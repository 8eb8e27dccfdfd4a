"""GPU tests of rm_page_slots, rm_paged_attention and rm_block_norm against the float64 oracle, alone and together.

Bounds (u32 = 2^-24 the unit roundoff of float32, u = that of the output type):
  slots:     whole numbers, equal.
  attention: |o - ref| <= u |ref| + (2 e (1 + e) + uP + (N + 32) u32) mag, mag the softmax average of |v|, uP = 2^-8 the
             rounding of the weights in bf16 (0 in float32), e a bound on a score's absolute error: the product's D + 8
             roundings of scale sum |q||k|, 4 roundings of the bias, and with a cap c the tanh's, 16 roundings of c.  A
             weight e^s is then off by at most e (1 + e) relatively, the sum of the weights too, hence 2 e.
  norm:      a sum of d squares is off by d u32 relatively at most, its root and the factor by r = (d / 2 + 8) u32; so
             u = x_scale x + f_scale gate f / rms gain is off by du <= (r + 8 u32) m, m = |x_scale x| + |the other term|,
             the norm of u relatively by (r + 8 u32) |m| / |u| (2-norms) and r, and out = u factor + shift by
             |factor| (du + |u| (r + (r + 8 u32) |m| / |u|)) + 8 u32 (|u factor| + |shift|), plus its own rounding."""
import numpy as np
import pytest
import torch

from oracle import attention as att
from oracle import serving

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_19104_amd as rm  # noqa: E402

U32 = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def gen(*path):
    g = torch.Generator()
    s = 23
    for p in path:
        s = s * 1000003 + int(p)
    g.manual_seed(s % (1 << 62))
    return g


def randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def ints(values):
    return torch.as_tensor(np.asarray(values), dtype=torch.int32).cuda()


# ----------------------------------------------------------------------------------------------------------
# Slots
# ----------------------------------------------------------------------------------------------------------

def check_slots(n_new, length, table, free, n_free, page, max_tok, in_place=False):
    """One call against the oracle; returns the oracle's step."""
    ref = serving.page_slots(n_new, length, table, free, n_free, page, max_tok)
    B = len(n_new)
    t = dict(n_new=ints(n_new), length=ints(length), table=ints(table), free_pages=ints(free), n_free=ints([n_free]))
    sizes = dict(first=B + 1, start=B, seq=max_tok, pos=max_tok, slot=max_tok, length_out=B, n_free_out=1, refused=1)
    # Each output between guards, filled with another value.
    bufs = {k: torch.full((n + 128,), -77, dtype=torch.int32, device="cuda") for k, n in sizes.items()}
    o = {k: bufs[k][64:64 + n] for k, n in sizes.items()}
    if in_place:
        o["length_out"], o["n_free_out"] = t["length"], t["n_free"]
    rm.rm_page_slots(t["n_new"], t["length"], t["table"], t["free_pages"], t["n_free"], o["first"], o["start"], o["seq"],
                     o["pos"], o["slot"], page, refused=o["refused"],
                     **({} if in_place else dict(length_out=o["length_out"], n_free_out=o["n_free_out"])))
    torch.cuda.synchronize()
    for name, want in (("first", ref.first), ("start", ref.start), ("seq", ref.seq), ("pos", ref.pos), ("slot", ref.slot),
                       ("length_out", ref.length), ("n_free_out", [ref.n_free]), ("refused", [ref.refused])):
        np.testing.assert_array_equal(o[name].cpu().numpy(), np.asarray(want), err_msg=name)
    np.testing.assert_array_equal(t["table"].cpu().numpy(), np.asarray(ref.table), err_msg="table")
    np.testing.assert_array_equal(t["free_pages"].cpu().numpy(), np.asarray(ref.free_pages), err_msg="free_pages")
    for k, n in sizes.items():
        b = bufs[k].cpu()
        assert (b[:64] == -77).all() and (b[64 + n:] == -77).all(), k
    return ref


@pytest.mark.parametrize("B,page,per,chunk,scarce", [
    (1, 1, 9, 4, False), (3, 16, 7, 40, False), (64, 16, 12, 1, False), (64, 7, 9, 20, True), (300, 8, 11, 30, False),
    (1024, 4, 5, 6, True), (1025, 16, 4, 3, False), (2500, 3, 5, 9, True), (2500, 64, 2, 70, False),
])
def test_steps_of_slots(B, page, per, chunk, scarce):
    """Several steps on the tables that the steps before them left."""
    rng = np.random.default_rng(B * 31 + page)
    n_pages = max(1, B * per // (4 if scarce else 1))
    length, table = [0] * B, rng.integers(-3, n_pages + 3, (B, per))
    free, n_free = rng.permutation(n_pages), n_pages
    for step in range(4):
        n_new = rng.integers(0, chunk + 1, B)
        n_new[rng.random(B) < 0.2] = -1
        n_new[rng.random(B) < 0.3] = 1
        max_tok = int(np.maximum(n_new, 0).sum()) + [0, 5, 1300, 0][step]
        r = check_slots(n_new, length, table, free, n_free, page, max(max_tok, 1), in_place=step % 2 == 1)
        length, table, free, n_free = r.length, r.table, r.free_pages, r.n_free


@pytest.mark.parametrize("n", [5000, 70001])
def test_slots_of_long_prompts(n):
    """Batches of many tokens: single long prompts, many short ones, requests without tokens between them."""
    rng = np.random.default_rng(n)
    for B, sizes in ((1, [n]), (7, [n - 60, 0, 3, 0, 50, 1, 6]), (600, [n // 600] * 600), (1500, None)):
        n_new = np.zeros(B, int) if sizes is None else np.asarray(sizes)
        if sizes is None:
            n_new[rng.integers(0, B, 40)] = n // 50
        page = 16
        per = -(-int(n_new.max()) // page) + 3
        n_pages = B * per
        length = rng.integers(0, 2 * page, B)
        perm = rng.permutation(n_pages)
        have = -(-length // page)
        table = np.where(np.arange(per) < have[:, None], perm.reshape(B, per), -1)
        free = np.concatenate((perm.reshape(B, per)[np.arange(per) >= have[:, None]], np.zeros(int(have.sum()), int)))
        check_slots(n_new, length, table, free, n_pages - int(have.sum()), page, n)
        check_slots(n_new, length, table, free, n_pages // 3, page, n - 100)  # too few pages, too little room


def test_slots_take_any_numbers():
    """Lengths, counts and tables that no step leaves."""
    big, low = (1 << 31) - 1, -(1 << 31)
    table = [[5, low, big], [-1, 3, 100], [0, 1, 2], [7, 8, 9], [9, 9, 9], [1, 2, 3]]
    free = [4, big, low, 6, 11, 3, 2, 1, 0, 5]
    for n_free in (low, 0, 4, big):
        for n_new in ([1] * 6, [big, big, 1, big, 0, 1], [low, -1, -1, 2, -1, 2], [big, big, big, 0, 0, 3], [0] * 6):
            for length in ([0, 4, big, low, 11, 12], [1, 5, 12, -1, 4, 3]):
                check_slots(n_new, length, table, free, n_free, 4, 7)


def test_slots_in_a_graph():
    """A decode loop captured once: lengths, tables and free pages stay on the GPU from replay to replay."""
    rng = np.random.default_rng(5)
    B, page, per = 37, 4, 6
    n_pages = B * per // 2
    length, table, free, n_free = rng.integers(0, 6, B), np.full((B, per), -1), rng.permutation(n_pages), n_pages
    r = serving.page_slots(length, [0] * B, table, free, n_free, page, 1000)
    length, table, free, n_free = r.length, r.table, r.free_pages, r.n_free
    t = dict(n_new=ints([1] * B), length=ints(length), table=ints(table), free_pages=ints(free), n_free=ints([n_free]))
    sizes = dict(first=B + 1, start=B, seq=B, pos=B, slot=B)
    o = {k: torch.zeros((n,), dtype=torch.int32, device="cuda") for k, n in sizes.items()}
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            rm.rm_page_slots(t["n_new"], t["length"], t["table"], t["free_pages"], t["n_free"], o["first"], o["start"],
                             o["seq"], o["pos"], o["slot"], page)
    for step in range(12):
        n_new = [-1 if rng.random() < 0.1 else 1 for _ in range(B)]
        t["n_new"].copy_(ints(n_new))
        graph.replay()
        torch.cuda.synchronize()
        r = serving.page_slots(n_new, length, table, free, n_free, page, B)
        for name, want in (("first", r.first), ("start", r.start), ("seq", r.seq), ("pos", r.pos), ("slot", r.slot)):
            np.testing.assert_array_equal(o[name].cpu().numpy(), np.asarray(want), err_msg=f"{name}, step {step}")
        np.testing.assert_array_equal(t["table"].cpu().numpy(), np.asarray(r.table))
        assert t["n_free"].item() == r.n_free and t["length"].tolist() == r.length
        length, table, free, n_free = r.length, r.table, r.free_pages, r.n_free


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,per,tokens,room", [
    (1, 16, 40, 257, 257), (1, 1, 9000, 8000, 8500), (3, 7, 30, 200, 700), (64, 16, 12, 30, 4097), (255, 3, 50, 60, 20000),
    (256, 24, 8, 40, 6000), (1000, 16, 4, 12, 9001), (1024, 8, 5, 9, 4100), (1024, 256, 2, 130, 100000),
])
def test_slots_by_many_workgroups(B, page, per, tokens, room, in_place):
    """Many tokens of up to 1024 requests: ended ones, scarce pages, too little room, requests that do not fit."""
    rng = np.random.default_rng(B + room)
    for scarce in (1.0, 0.3):
        n_pages = max(2, int(B * per * scarce))
        length, table, free, n_free = [0] * B, rng.integers(-3, n_pages + 3, (B, per)), rng.permutation(n_pages), n_pages
        for step in range(5):
            n_new = rng.integers(0, tokens + 1, B)
            n_new[rng.random(B) < 0.25] = -1
            n_new[rng.random(B) < 0.2] = 1
            n_new[rng.random(B) < 0.02] = per * page + 1
            if step == 0:
                n_new[0] = tokens
            r = check_slots(n_new, length, table, free, n_free, page, room, in_place=in_place)
            length, table, free, n_free = r.length, r.table, r.free_pages, r.n_free


def test_slots_by_many_workgroups_in_a_graph():
    """Prompts captured once and replayed, with the lengths, the count, both or neither updated in place."""
    rng = np.random.default_rng(6)
    B, page, per, room = 90, 8, 16, 5000
    n_pages = B * per // 3
    for length_out, n_free_out in ((None, None), (B, None), (None, 1), (B, 1)):
        length, table, free, n_free = [0] * B, np.full((B, per), -1), rng.permutation(n_pages), n_pages
        t = dict(n_new=ints([0] * B), length=ints(length), table=ints(table), free_pages=ints(free), n_free=ints([n_free]))
        sizes = dict(first=B + 1, start=B, seq=room, pos=room, slot=room)
        o = {k: torch.zeros((n,), dtype=torch.int32, device="cuda") for k, n in sizes.items()}
        told = [None if n is None else torch.zeros((n,), dtype=torch.int32, device="cuda") for n in (length_out, n_free_out)]
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                rm.rm_page_slots(t["n_new"], t["length"], t["table"], t["free_pages"], t["n_free"], o["first"], o["start"],
                                 o["seq"], o["pos"], o["slot"], page, length_out=told[0], n_free_out=told[1])
        for step in range(6):
            n_new = rng.integers(0, 60, B)
            n_new[rng.random(B) < 0.3] = -1
            t["n_new"].copy_(ints(n_new))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            r = serving.page_slots(n_new, length, table, free, n_free, page, room)
            for name, want in (("first", r.first), ("start", r.start), ("seq", r.seq), ("pos", r.pos), ("slot", r.slot)):
                np.testing.assert_array_equal(o[name].cpu().numpy(), np.asarray(want), err_msg=f"{name}, step {step}")
            for name, own, want in (("length", told[0], r.length), ("n_free", told[1], [r.n_free])):
                np.testing.assert_array_equal((t[name] if own is None else own).cpu().numpy(), np.asarray(want))
                if own is not None:
                    t[name].copy_(own)
            np.testing.assert_array_equal(t["table"].cpu().numpy(), np.asarray(r.table))
            np.testing.assert_array_equal(t["free_pages"].cpu().numpy(), np.asarray(r.free_pages))
            length, table, free, n_free = r.length, r.table, r.free_pages, r.n_free


# ----------------------------------------------------------------------------------------------------------
# Paged attention
# ----------------------------------------------------------------------------------------------------------

def attention_bound(ref, mag, big, dtype, D, n, cap=0.0, bias=0.0):
    e = (D + 8) * U32 * big[..., None] + 4 * U32 * bias + (16 * U32 * cap if cap else 0.0)
    up = 2.0 ** -8 if dtype == BF else 0.0
    return U[dtype] * np.abs(ref) + (2 * e * (1 + e) + up + (n + 32) * U32) * mag + 1e-30


def run_paged(q, k, v, table, pos, seq=None, window=0, slopes=None, scale=None, cap=0.0, out=None):
    if out is None:
        out = torch.full_like(q, NAN)
    ws = rm.paged_attention_workspace(q, k, table)
    ws.fill_(0xFF)
    rm.rm_paged_attention(q, k, v, table, pos, out, ws, seq=seq, window=window, slopes=slopes, scale=scale, softcap=cap)
    torch.cuda.synchronize()
    return out


def check_paged(q, k, v, table, pos, seq=None, window=0, slopes=None, scale=None, cap=0.0, out=None, heads=None):
    D = q.shape[2]
    if out is None:
        out = run_paged(q, k, v, table, pos, seq, window, slopes, scale, cap)
    s = D ** -0.5 if scale is None else scale
    ref, mag, big = serving.paged_attention(f64(q), f64(k), f64(v), table.cpu().numpy(),
                                            None if seq is None else seq.cpu().numpy(), pos.cpu().numpy(), window,
                                            np.float32(s), cap, f64(slopes), heads)
    longest = int(pos.max().clamp(0, table.shape[1] * k.shape[1])) + 1
    bias = 0.0 if slopes is None else float(slopes.abs().max()) * (int(pos.max()) + 1)
    tol = attention_bound(ref, mag, big, q.dtype, D, longest, cap, bias)
    got = f64(out)
    if heads is not None:
        got, ref, tol = got[:, heads], ref[:, heads], tol[:, heads]
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"error {float((err / tol).max()):.3f} times the bound"
    return out


def cache(g, N, per, page, Hk, D, dtype, spare=3):
    n_pages = N * per + spare
    table = torch.randperm(n_pages, generator=g)[:N * per].to(torch.int32).view(N, per).cuda()
    return randn(g, (n_pages, page, Hk, D), dtype), randn(g, (n_pages, page, Hk, D), dtype), table


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 128, 136, 200, 256])
@pytest.mark.parametrize("page", [1, 16, 24, 256])
def test_paged(dtype, D, page):
    """Positions around the ends of pages and tiles, heads of every kernel's width."""
    g = gen(1, D, page, dtype == BF)
    pos = ints([0, 1, 14, 15, 16, 17, 31, 32, 63, 64, 65, 127, 128, 129, 200, 299])
    N = len(pos)
    k, v, table = cache(g, N, -(-300 // page), page, 2, D, dtype)
    check_paged(randn(g, (N, 4, D), dtype, 2.0), k, v, table, pos)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (7, 1), (16, 1), (17, 1), (32, 1), (33, 1), (40, 1), (71, 1), (12, 2)])
def test_paged_head_layouts(dtype, D, Hq, Hk):
    g = gen(2, Hq, Hk, D)
    pos = ints([0, 77, 139, 260])
    k, v, table = cache(g, 4, 9, 32, Hk, D, dtype)
    check_paged(randn(g, (4, Hq, D), dtype, 2.0), k, v, table, pos)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap,bias,window", [(30.0, False, 0), (0.0, True, 0), (5.0, True, 0), (0.0, False, 1),
                                             (0.0, False, 100), (20.0, True, 33), (300.0, False, 0), (1e6, True, 77)])
@pytest.mark.parametrize("D", [72, 128, 256])
def test_paged_cap_bias_window(dtype, cap, bias, window, D):
    g = gen(3, int(cap), bias, window, D)
    pos = ints([0, 5, 99, 100, 101, 333, 500])
    k, v, table = cache(g, 7, 32, 16, 2, D, dtype)
    slopes = torch.tensor([0.5, 0.1, 0.0, 0.03, 0.01, 0.2], device="cuda") if bias else None
    check_paged(randn(g, (7, 6, D), dtype, 2.0), k, v, table, pos, window=window, slopes=slopes, cap=cap)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_paged_bias_far_behind_the_table(dtype, cap):
    """Positions far behind the table's last key add the same to a head's scores, slope times the rest of the distance, and
    so leave its weights as they are at the last key's position."""
    g = gen(17)
    N, Hq, Hk, D, page, per = 6, 8, 2, 64, 16, 7
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    q = randn(g, (N, Hq, D), dtype, 2.0)
    slopes = (torch.rand((Hq,), generator=g) * 0.3 + 0.05).cuda()
    far = run_paged(q, k, v, table, ints([page * per, 1 << 20, (1 << 24) + 1, 1 << 28, (1 << 30) + 7, (1 << 31) - 1]),
                    slopes=slopes, cap=cap)
    check_paged(q, k, v, table, ints([page * per - 1] * N), slopes=slopes, cap=cap, out=far)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,Hq,Hk,N,length", [(64, 8, 1, 1, 20000), (128, 8, 2, 3, 9000), (256, 8, 1, 1, 5000),
                                              (72, 4, 4, 2, 3001), (128, 40, 1, 2, 4000)])
def test_long_caches(dtype, D, Hq, Hk, N, length):
    """Keys that several workgroups divide."""
    g = gen(4, D, N)
    page = 16
    k, v, table = cache(g, N, -(-length // page), page, Hk, D, dtype)
    pos = ints([length - 1 - 37 * i for i in range(N)])
    check_paged(randn(g, (N, Hq, D), dtype, 2.0), k, v, table, pos, heads=[0, Hq // 2, Hq - 1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,Hq,Hk", [(128, 8, 4), (64, 6, 6), (256, 2, 1)])
@pytest.mark.parametrize("N", [63, 64, 65, 400])
def test_ragged_batches(dtype, D, Hq, Hk, N):
    """Many requests of lengths from nothing to long, in another order than the tables."""
    g = gen(5, D, N)
    page, per = 16, 40
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    pos = (torch.rand((N,), generator=g) ** 3 * per * page).to(torch.int32)
    pos[::9] = -1
    pos[4] = per * page - 1
    seq = torch.randperm(N, generator=g).to(torch.int32).cuda()
    check_paged(randn(g, (N, Hq, D), dtype, 2.0), k, v, table, pos.cuda(), seq=seq, heads=[0, Hq - 1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 72, 128, 256])
def test_paged_unseen_rows_may_hold_anything(dtype, D):
    """NaN and infinities in every row that no token sees, on pages that are none, and before the window."""
    g = gen(6, D)
    N, per, page, Hk, Hq = 6, 12, 16, 2, 8
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    pos, window = [0, 20, 100, 191, 47, 48], 90
    host = table.cpu()
    seen = torch.zeros((k.shape[0], page), dtype=torch.bool)
    bad = [(2, 4), (3, 10), (5, 0)]
    for n, p in enumerate(pos):
        for j in range(max(0, p - window + 1), p + 1):
            if (n, j // page) not in bad:
                seen[host[n, j // page], j % page] = True
    for i, (n, pg) in enumerate(bad):
        host[n, pg] = [-1, k.shape[0], (1 << 31) - 1][i]
    for fill in (NAN, float("inf"), -float("inf")):
        kk, vv = k.clone(), v.clone()
        kk[~seen.cuda()] = fill
        vv[~seen.cuda()] = fill
        a = check_paged(q := randn(gen(7, D), (N, Hq, D), dtype, 2.0), kk, vv, host.cuda(), ints(pos), window=window)
        assert torch.equal(a, run_paged(q, k, v, host.cuda(), ints(pos), window=window))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_tokens_that_see_nothing(dtype):
    g = gen(8)
    D = 64
    k, v, table = cache(g, 3, 4, 16, 1, D, dtype)
    q = randn(g, (8, 4, D), dtype)
    seq = ints([0, 3, -1, 1, (1 << 31) - 1, -(1 << 31), 2, 2])
    pos = ints([-1, 5, 5, -(1 << 31), 0, 3, 63, 30])
    out = check_paged(q, k, v, table, pos, seq=seq)
    assert (out[:6] == 0).all() and (out[6:] != 0).any(-1).all()
    far = ints([64, (1 << 31) - 1, 1000, 66, 63, 70, 64, 65])  # past the table: its last key is the last one
    seq = ints([0, 1, 2, 0, 1, 2, 0, 1])
    check_paged(q, k, v, table, far, seq=seq)
    check_paged(q, k, v, table, far, seq=seq, window=7)
    k[:] = NAN
    out = run_paged(q, k, v, torch.full_like(table, -1), ints([40] * 8), seq=seq)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_without_end(dtype, D):
    """A key whose score is -infinity has no weight, a token whose scores all are gives 0; an infinite value that is seen
    comes through; a score of +infinity or NaN gives NaN in its head alone."""
    g = gen(9, D)
    k, v, table = cache(g, 3, 6, 16, 2, D, dtype)
    q = randn(g, (3, 4, D), dtype, 2.0)
    q[..., 0] = q[..., 0].abs() + 0.5
    pos = ints([60, 90, 7])
    page = table[0, 1].item()
    k[page, 3, 0, 0] = -float("inf")  # key 19 of request 0, head 0
    out = run_paged(q, k, v, table, pos)
    k2 = k.clone()
    k2[page, 3, 0, :] = 0
    ref = serving.paged_attention(f64(q), f64(k2), f64(v), table.cpu().numpy(), None, pos.cpu().numpy(), 0,
                                  np.float32(D ** -0.5))[0]
    kk, vv = f64(k2)[table.cpu()[0]].reshape(-1, 2, D)[:61, 0], f64(v)[table.cpu()[0]].reshape(-1, 2, D)[:61, 0]
    seen = np.ones((1, 61), bool)
    seen[0, 19] = False
    for h in (0, 1):
        ref[0, h] = att.attend(f64(q)[0, h:h + 1], kk, vv, seen, np.float32(D ** -0.5), 0.0, None)[0][0]
    np.testing.assert_allclose(f64(out), ref, rtol=0, atol=0.03 if dtype == BF else 1e-4)
    k[table[2, 0].item(), :8, :, 0] = -float("inf")
    assert (run_paged(q, k, v, table, pos)[2] == 0).all()
    v[table[1, 2].item(), 5, 1, 7] = float("inf")
    out = run_paged(q, k, v, table, pos)
    assert (out[1, 2:, 7] == float("inf")).all() and out[1].isinf().sum() == 2
    k[table[1, 0].item(), 5, 0, 0] = float("inf")
    out = run_paged(q, k, v, table, pos)
    assert out[1, :2].isnan().all() and not out[1, 2:].isnan().any() and not out[0].isnan().any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_paged_strides(dtype):
    """Keys beside values in a cache row, pages that hold one head after the other, queries and outputs inside the rows of
    wider tensors; nothing beside the output is written."""
    g = gen(10)
    N, Hq, Hk, D, page, per = 5, 6, 2, 72, 8, 9
    n_pages = N * per + 1
    table = torch.randperm(n_pages, generator=g)[:N * per].to(torch.int32).view(N, per).cuda()
    pos = ints([0, 70, 33, 8, 55])
    qkv = randn(g, (N, Hq + 4, D + 8), dtype)
    q = qkv[:, 2:2 + Hq, 8:]
    both = randn(g, (n_pages, page, 2, Hk, D), dtype)
    by_head = randn(g, (n_pages, Hk, page, D), dtype).permute(0, 2, 1, 3)
    shared = randn(g, (1, page, Hk, D), dtype).expand(n_pages, page, Hk, D)
    for k, v in ((both[:, :, 0], both[:, :, 1]), (by_head, both[:, :, 1]), (both[:, :, 0], by_head), (shared, by_head)):
        wide = torch.full((N, Hq + 3, D + 16), 7.0, dtype=dtype, device="cuda")
        out = wide[:, 1:1 + Hq, 8:8 + D]
        run_paged(q, k, v, table, pos, out=out)
        check_paged(q, k, v, table, pos, out=out)
        out.fill_(7.0)
        assert (wide == 7.0).all()


def test_paged_offsets_past_32_bits():
    """A cache of 5 GB, its last pages among those in use."""
    g = gen(11)
    page, Hk, D, per = 64, 8, 128, 40
    n_pages = 5 * (1 << 30) // (page * Hk * D * 2)
    k = torch.zeros((n_pages, page, Hk, D), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    table = torch.randperm(n_pages, generator=g)[:2 * per].to(torch.int32).view(2, per)
    table[0, 3], table[1, per - 1], table[1, 0] = n_pages - 1, n_pages - 2, 0
    used = table.flatten().long().cuda()
    k[used], v[used] = randn(g, (2 * per, page, Hk, D), BF), randn(g, (2 * per, page, Hk, D), BF)
    q, pos = randn(g, (2, 16, D), BF, 2.0), ints([per * page - 1, per * page - 3])
    out = run_paged(q, k, v, table.cuda(), pos)
    compact = torch.arange(2 * per, dtype=torch.int32).view(2, per).cuda()
    check_paged(q, k[used], v[used], compact, pos, out=out, heads=[0, 7, 15])


def test_paged_offsets_past_36_bits():
    """Pages 40 GiB apart: more than 2^32 pieces of 16 bytes."""
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GiB of free memory")
    g = gen(15)
    page, Hk, D = 16, 2, 64
    apart = (40 << 30) // 2
    room = torch.empty((2 * apart + page * Hk * D * 2,), dtype=BF, device="cuda")
    k = room.as_strided((3, page, Hk, D), (apart, Hk * D, D, 1))
    v = room.as_strided((3, page, Hk, D), (apart, Hk * D, D, 1), page * Hk * D)
    near_k, near_v = randn(g, (3, page, Hk, D), BF), randn(g, (3, page, Hk, D), BF)
    k.copy_(near_k)
    v.copy_(near_v)
    table, pos, q = ints([[2, 0, 1], [1, 2, 0]]), ints([40, 17]), randn(g, (2, 8, D), BF, 2.0)
    out = run_paged(q, k, v, table, pos)
    check_paged(q, near_k, near_v, table, pos, out=out)
    assert torch.equal(out, run_paged(q, near_k, near_v, table, pos))
    del room, k, v
    torch.cuda.empty_cache()


def test_paged_batches_of_one_wave():
    """So few keys that no token is divided: no workspace."""
    g = gen(16)
    for N, D, Hq, Hk, dtype in ((1, 64, 8, 1, BF), (1, 128, 80, 2, F32), (2, 72, 4, 4, BF)):
        k, v, table = cache(g, N, 2, 16, Hk, D, dtype)
        q = randn(g, (N, Hq, D), dtype, 2.0)
        assert rm.paged_attention_workspace(q, k, table).numel() == 0 or N * 2 * 16 > 32
        for p in (0, 13, 31):
            check_paged(q, k, v, table, ints([p - i for i in range(N)]))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_paged_is_the_same_on_every_call(dtype):
    """Repeated calls, with other things in the workspace, on another stream, and captured and replayed on new positions."""
    g = gen(12)
    N, Hq, Hk, D, page, per = 9, 8, 2, 128, 16, 150
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    q = randn(g, (N, Hq, D), dtype, 2.0)
    places = [ints([int(x) for x in torch.randint(-1, per * page, (N,), generator=g)]) for _ in range(5)]
    eager = [run_paged(q, k, v, table, p) for p in places]
    check_paged(q, k, v, table, places[0], out=eager[0], heads=[0, 5])
    pos, out = places[0].clone(), torch.zeros_like(q)
    ws = rm.paged_attention_workspace(q, k, table)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    rm.rm_paged_attention(q, k, v, table, pos, out, ws, stream=s)
    s.synchronize()
    assert torch.equal(out, eager[0])
    with torch.cuda.stream(s):
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]  # which share the workspace
        for graph in graphs:
            with torch.cuda.graph(graph, stream=s):
                rm.rm_paged_attention(q, k, v, table, pos, out, ws)
    for i, p in enumerate(places):
        pos.copy_(p)
        ws.fill_(0xFF)
        out.fill_(NAN)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i])


def test_several_tokens_of_a_request():
    """A request's chunk of tokens, each at its position on the same table, is causal attention."""
    g = gen(13)
    Hq, Hk, D, page, per, T = 8, 2, 64, 16, 8, 37
    k, v, table = cache(g, 2, per, page, Hk, D, BF)
    seq = ints([1] * T + [0] * 3)
    pos = ints(list(range(60, 60 + T)) + [3, 4, 5])
    check_paged(randn(g, (T + 3, Hq, D), BF, 2.0), k, v, table, pos, seq=seq)


def test_paged_refuses_a_small_workspace_and_other_devices():
    g = gen(14)
    k, v, table = cache(g, 2, 600, 16, 1, 128, BF)
    q = randn(g, (2, 8, 128), BF)
    n = rm.paged_attention_workspace(q, k, table).numel()
    pos = ints([9000, 9000])
    if n > 0:
        with pytest.raises(rm.RmError) as e:
            rm.rm_paged_attention(q, k, v, table, pos, torch.empty_like(q),
                                  torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
        assert e.value.status == rm.RM_ERR_WORKSPACE
    with pytest.raises(ValueError):
        rm.rm_paged_attention(q, k.cpu(), v, table, pos, torch.empty_like(q), None)
    with pytest.raises(ValueError):
        rm.rm_paged_attention(q, k, v, table.long(), pos, torch.empty_like(q), None)
    with pytest.raises(ValueError):
        rm.rm_paged_attention(q, k, v, table, pos[:1], torch.empty_like(q), None)
    with pytest.raises(ValueError):
        rm.rm_paged_attention(q, k, v.float(), table, pos, torch.empty_like(q), None)


# ----------------------------------------------------------------------------------------------------------
# Block norm
# ----------------------------------------------------------------------------------------------------------

def norm_bounds(ref, shift, d, yt, ot):
    """Tolerances of y and out."""
    r = (d / 2 + 8) * U32
    du = (r + 8 * U32) * ref.mag
    size = lambda a: np.sqrt((a * a).sum(-1, keepdims=True))  # noqa: E731
    rel = r + (r + 8 * U32) * size(ref.mag) / np.maximum(size(ref.y), 1e-300)
    s = 0.0 if shift is None else np.abs(shift)[:, None]
    do = np.abs(ref.factor) * (du + np.abs(ref.y) * rel) + 8 * U32 * (np.abs(ref.y * ref.factor) + s)
    return U[yt] * np.abs(ref.y) + (1 + U[yt]) * du + 1e-38, U[ot] * np.abs(ref.out) + (1 + U[ot]) * do + 1e-38


def check_norm(x, f, y, out, **kw):
    x0, f0 = x.clone(), None if f is None else f.clone()  # (y may be x, out may be f)
    rm.rm_block_norm(x, f, y, out, **kw)
    torch.cuda.synchronize()
    args = {k: f64(a) if isinstance(a, torch.Tensor) else a for k, a in kw.items()}
    for k in ("x_scale", "f_scale", "eps"):
        if k in args:
            args[k] = float(np.float32(args[k]))
    args.setdefault("norm_post", False)
    args.setdefault("eps", float(np.float32(1e-6)))
    ref = serving.block_norm(f64(x0), f64(f0), **args)
    ty, to = norm_bounds(ref, args.get("shift"), x.shape[-1], x.dtype, F32 if out is None else out.dtype)
    for name, got, want, tol in (("y", y, ref.y, ty), ("out", out, ref.out, to)):
        if got is not None:
            err = np.abs(f64(got) - want)
            assert (err <= tol).all(), f"{name}: error {float((err / tol).max()):.3f} times the bound"


@pytest.mark.parametrize("xt", [F32, BF])
@pytest.mark.parametrize("ft", [F32, BF])
@pytest.mark.parametrize("ot", [F32, BF])
@pytest.mark.parametrize("d", [8, 264, 1024, 2048])
def test_block_norm_types(xt, ft, ot, d):
    g = gen(20, xt == BF, ft == BF, ot == BF, d)
    B, T = 3, 17
    x, f = randn(g, (B, T, d), xt, 2.0), randn(g, (B, T, d), ft)
    mod = randn(g, (B, 3 * d), F32, 0.3)
    check_norm(x, f, torch.full_like(x, NAN), torch.full_like(x, NAN, dtype=ot), norm_post=True,
               gain_post=randn(g, (d,), F32), gate=mod[:, 2 * d:], gain_pre=randn(g, (d,), F32), scale=mod[:, :d],
               shift=mod[:, d:2 * d], x_scale=0.7, f_scale=-1.3, eps=1e-5)


@pytest.mark.parametrize("which", range(10))
@pytest.mark.parametrize("rows", [(1, 1), (2, 51), (1, 3000)])
def test_block_norm_parts(which, rows):
    """Every part left out by itself, alone, and both ends of a stack."""
    d = 320
    g = gen(21, which, *rows)
    B, T = rows
    x, f = randn(g, (B, T, d), F32, 2.0), randn(g, (B, T, d), BF)
    y, out = torch.full_like(x, NAN), torch.full_like(x, NAN, dtype=BF)
    vec, mod = (lambda: randn(g, (d,), F32)), (lambda: randn(g, (B, d), F32))
    if which == 0:
        check_norm(x, f, y, out)
    elif which == 1:
        check_norm(x, f, y, None, norm_post=True, gain_post=vec(), gate=mod())
    elif which == 2:
        check_norm(x, None, None, out, gain_pre=vec(), scale=mod(), shift=mod())
    elif which == 3:
        check_norm(x, None, y, out, scale=mod(), x_scale=2.0)
    elif which == 4:
        check_norm(x, f, None, out, shift=mod())
    elif which == 5:
        check_norm(x, f, y, out, norm_post=True)
    elif which == 6:
        check_norm(x, f, x, out, gate=mod())                        # in place
    elif which == 7:
        check_norm(x, f, y, f, norm_post=True, gain_post=vec(), gain_pre=vec())  # the output over the block's
    elif which == 8:
        check_norm(x, f, x, f, norm_post=True, gate=mod(), scale=mod(), shift=mod())
    else:
        check_norm(x, f, x, None, f_scale=0.0)


@pytest.mark.parametrize("d", [8, 16, 512, 520, 1152, 2056, 4096, 8192, 8200, 16384, 32768])
@pytest.mark.parametrize("T", [1, 5, 2500])
def test_block_norm_widths(d, T):
    if d * T > 1 << 24:
        T = (1 << 24) // d
    g = gen(22, d, T)
    x, f = randn(g, (2, T, d), BF, 2.0), randn(g, (2, T, d), BF)
    buf = torch.full((2 * T * d + 64,), 7.0, dtype=BF, device="cuda")
    out = buf[32:32 + 2 * T * d].view(2, T, d)
    check_norm(x, f, torch.full_like(x, NAN), out, norm_post=True, gain_post=randn(g, (d,), F32), gate=randn(g, (2, d), F32),
               gain_pre=randn(g, (d,), F32), scale=randn(g, (2, d), F32), shift=randn(g, (2, d), F32))
    assert (buf[:32] == 7.0).all() and (buf[-32:] == 7.0).all()


def test_block_norm_extremes():
    """Rows of zeros, tiny and large rows, and rows with infinities or NaN, which stay in their rows."""
    d = 256
    g = gen(23)
    x, f = randn(g, (1, 9, d), F32), randn(g, (1, 9, d), F32)
    x[0, 0], f[0, 0] = 0, 0
    x[0, 1] *= 1e-20
    f[0, 1] *= 1e-20
    x[0, 2] *= 1e15
    f[0, 3] *= 1e15
    y, out = torch.full_like(x, NAN), torch.full_like(x, NAN)
    check_norm(x, f, y, out, norm_post=True)
    assert (out[0, 0] == 0).all()
    z, o = y.clone(), out.clone()
    x[0, 4, 7] = float("inf")
    f[0, 5, 3] = NAN
    rm.rm_block_norm(x, f, y, out, norm_post=True)
    torch.cuda.synchronize()
    keep = [0, 1, 2, 3, 6, 7, 8]
    assert torch.equal(y[0, keep], z[0, keep]) and torch.equal(out[0, keep], o[0, keep])
    assert y[0, 4, 7] == float("inf") and out[0, 4, 7].isnan() and out[0, 5].isnan().all()


# ----------------------------------------------------------------------------------------------------------
# Together
# ----------------------------------------------------------------------------------------------------------

def test_decode_steps_of_a_layer():
    """Steps of one layer's attention side as a server makes them, captured once and replayed: slots, norm and rotation
    into the pages, attention over them, and the passage to the next block.  Prompts come first, then single tokens, while
    requests end and others begin in their place; the oracle keeps its own cache."""
    g = gen(30)
    rng = np.random.default_rng(30)
    B, Hq, Hk, D, page, per, d, M = 6, 4, 2, 64, 8, 12, 256, 60
    n_pages = B * per
    dev = dict(device="cuda")
    inv_freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    gain = randn(g, (d,), F32)
    w_out = randn(g, (Hq * D, d), F32, 0.05).to(BF)
    k_cache = torch.full((n_pages, page, Hk, D), NAN, dtype=BF, **dev)
    v_cache = torch.full_like(k_cache, NAN)
    n_new, length = torch.zeros(B, dtype=torch.int32, **dev), torch.zeros(B, dtype=torch.int32, **dev)
    table = torch.full((B, per), -1, dtype=torch.int32, **dev)
    free, n_free = ints(rng.permutation(n_pages)), ints([n_pages])
    first, start = torch.zeros(B + 1, dtype=torch.int32, **dev), torch.zeros(B, dtype=torch.int32, **dev)
    seq, pos, slot = (torch.zeros(M, dtype=torch.int32, **dev) for _ in range(3))
    qkv = torch.zeros((M, Hq + 2 * Hk, D), dtype=BF, **dev)
    x = torch.zeros((1, M, d), **dev)
    q_out, att_out = (torch.zeros((M, Hq, D), dtype=BF, **dev) for _ in range(2))
    y, out, f = torch.zeros_like(x), torch.zeros_like(x), torch.zeros((1, M, d), dtype=BF, **dev)
    ws = rm.paged_attention_workspace(q_out, k_cache, table)

    def step():
        rm.rm_page_slots(n_new, length, table, free, n_free, first, start, seq, pos, slot, page)
        rm.rm_qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], q_out, k_cache.view(-1, Hk, D),
                           v_cache.view(-1, Hk, D), pos, inv_freq, slot=slot)
        rm.rm_paged_attention(q_out, k_cache, v_cache, table, pos, att_out, ws, seq=seq)
        torch.mm(att_out.view(M, Hq * D), w_out, out=f[0])
        rm.rm_block_norm(x, f, y, out, norm_post=True, gain_post=gain)

    state = [n_new, length, table, free, n_free]
    keep = [t.clone() for t in state]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()  # (the library product's own preparations)
        s.synchronize()
        for t, k in zip(state, keep):
            t.copy_(k)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.synchronize()
    told = dict(length=[0] * B, table=np.full((B, per), -1), free=free.cpu().numpy(), n_free=n_pages)
    rows = [[] for _ in range(B)]  # every request's (k, v) so far, as the cache rounds them
    for i in range(14):
        new = [int(rng.integers(3, 15)) if n == 0 and rng.random() < 0.7 else 1 if n > 0 else 0 for n in told["length"]]
        new = [-1 if told["length"][b] > 0 and rng.random() < 0.12 else n for b, n in enumerate(new)]
        n_new.copy_(ints(new))
        qkv.copy_(randn(g, qkv.shape, BF, 2.0))
        x.copy_(randn(g, x.shape, F32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r = serving.page_slots(new, told["length"], told["table"], told["free"], told["n_free"], page, M)
        for name, got, want in (("seq", seq, r.seq), ("pos", pos, r.pos), ("slot", slot, r.slot), ("length", length, r.length)):
            np.testing.assert_array_equal(got.cpu().numpy(), np.asarray(want), err_msg=f"{name}, step {i}")
        told = dict(length=r.length, table=r.table, free=r.free_pages, n_free=r.n_free)
        for b in range(B):
            if new[b] < 0:
                rows[b] = []
        p = np.maximum(np.asarray(r.pos), 0)
        turned = att.norm_rope(f64(qkv)[:, Hq:Hq + Hk], None, p, f64(inv_freq), 1e-6, False)
        kc, vc = f64(k_cache).reshape(-1, Hk, D), f64(v_cache).reshape(-1, Hk, D)
        for t in range(M):
            if r.slot[t] >= 0:
                # A rotated pair of bf16 in bf16: half a step of its length, and the angle's error.
                assert np.abs(kc[r.slot[t]] - turned[t]).max() <= (2.0 ** -8 + 2.0 ** -20) * np.abs(turned[t]).max() * 1.5
                assert np.array_equal(vc[r.slot[t]], f64(qkv)[t, Hq + Hk:])
                rows[r.seq[t]].append((kc[r.slot[t]], vc[r.slot[t]]))
        # Earlier rows are still what they were, and the attention is that of the request's own rows.
        qd = f64(q_out)
        for t in range(M):
            if r.pos[t] < 0:
                assert (att_out[t] == 0).all()
                continue
            ks, vs = (np.stack([a[j] for a in rows[r.seq[t]][:r.pos[t] + 1]]) for j in (0, 1))
            at = [r.table[r.seq[t]][j // page] * page + j % page for j in range(r.pos[t] + 1)]
            assert np.array_equal(kc[at], ks) and np.array_equal(vc[at], vs)
            for h in range(Hq):
                o, m, b = att.attend(qd[t, h:h + 1], ks[:, h // 2], vs[:, h // 2], np.ones((1, len(at)), bool),
                                     np.float32(D ** -0.5), 0.0, None)
                assert (np.abs(f64(att_out)[t, h] - o[0]) <= attention_bound(o, m, b, BF, D, len(at))[0]).all()
        ref = serving.block_norm(f64(x), f64(f), True, gain_post=f64(gain), eps=float(np.float32(1e-6)))
        ty, to = norm_bounds(ref, None, d, F32, F32)
        assert (np.abs(f64(y) - ref.y) <= ty).all() and (np.abs(f64(out) - ref.out) <= to).all()
