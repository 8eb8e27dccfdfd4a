"""GPU tests of the serving-step calls where their bounds are tight: weights of bf16 attention, biases far from their zero, caps
of every size, batches past 512 tokens; and block norms past one launch.

Bound (u32 = 2^-24, u = the output type's half step): as in test_gpu_serving.py, with the weights in two bf16 parts: the
first by truncation, which leaves a rest below 2^-7 of the weight, the second the rest rounded by at most 2^-8 of it, so a
weight is off by 2^-15.  A bound is worth its name while it leaves little beside the output's own rounding: of every case the
rest is at most `spare` of the softmax average of |v|, and most values are four bounds from 0 or more."""
import numpy as np
import pytest
import torch

import paper_2609_19104_amd as rm
from oracle import serving

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_serving import BF, F32, U, U32, cache, f64, gen, ints, randn, run_paged  # noqa: E402


def paged_within(out, q, k, v, table, pos, e, spare, seq=None, window=0, slopes=None, scale=None, cap=0.0, heads=None,
                 counted=None):
    """out against the oracle, e(big) the bound of a score's error, big the score's size sum |q||k| scale; counted: keys whose
    weights are not too small to change the sums."""
    D = q.shape[2]
    s = np.float32(D ** -0.5 if scale is None else scale)
    ref, mag, big = serving.paged_attention(f64(q), f64(k), f64(v), table.cpu().numpy(),
                                            None if seq is None else seq.cpu().numpy(), pos.cpu().numpy(), window, s, cap,
                                            f64(slopes), heads)
    longest = min(int(pos.max()) + 1, table.shape[1] * k.shape[1]) if counted is None else counted
    x = e(big[..., None])
    rest = 2 * x * (1 + x) + (2.0 ** -15 if q.dtype == BF else 0.0) + (longest + 32) * U32
    got, at = f64(out), slice(None) if heads is None else heads
    assert rest[:, at].max() <= spare
    tol = (U[q.dtype] * np.abs(ref) + (1 + U[q.dtype]) * rest * mag + 1e-30)[:, at]
    seen = mag[:, at] > 0  # (a bound that most values lie within says nothing)
    assert (4 * tol[seen] < np.abs(ref[:, at])[seen]).mean() > 0.5
    err = np.abs(got - ref)[:, at]
    assert np.isfinite(got).all()
    assert (err <= tol).all(), f"error {float((err / tol).max()):.3f} times the bound"


# ----------------------------------------------------------------------------------------------------------
# Weights
# ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("D,Hq,Hk", [(64, 8, 1), (72, 6, 3), (96, 16, 1), (128, 20, 1), (192, 4, 2), (256, 8, 1)])
@pytest.mark.parametrize("length", [2, 40, 300, 5000])
def test_weights_of_bf16_keep_their_digits(D, Hq, Hk, length):
    """The output of bf16 values is as exact as its own rounding: weights lose 2^-15 where one bf16 number a weight would lose
    2^-8.  Scores are small (about 1), so that their own error is too."""
    g = gen(40, D, length)
    N, page = 3, 16
    k, v, table = cache(g, N, -(-length // page), page, Hk, D, BF)
    q, pos = randn(g, (N, Hq, D), BF), ints([length - 1, length // 2, length - 1 - length // 7])
    # scale sum |q||k| is up to about 0.64 D / sqrt(D) and some: 14 at 256 columns, 2 e 0.0005 at most.
    paged_within(run_paged(q, k, v, table, pos), q, k, v, table, pos, lambda big: (D + 8) * U32 * big, 2.0 ** -10,
                 heads=[0, Hq - 1])


@pytest.mark.parametrize("low", [0.0, 20.0, 60.0, 68.0])
def test_small_weights_of_infinite_values(low):
    """A seen infinite value comes through under any weight that is not 0, also where its weight is one bf16 number."""
    g = gen(41, int(low))
    D, page = 64, 16
    k, v, table = cache(g, 1, 4, page, 1, D, BF)
    k[:] = 0
    q = torch.zeros((1, 8, D), dtype=BF, device="cuda")
    q[..., 0] = 1.0
    at = table[0, 2].item()
    k[at, 5, 0, 0] = -low  # scores 0, and one of -low
    v[at, 5, 0, 9] = float("inf")
    v[at, 5, 0, 20] = -float("inf")
    out = run_paged(q, k, v, table, ints([63]), scale=1.0)
    assert (out[..., 9] == float("inf")).all() and (out[..., 20] == -float("inf")).all()
    keep = [c for c in range(D) if c not in (9, 20)]
    assert out[..., keep].isfinite().all()


# ----------------------------------------------------------------------------------------------------------
# Block norm
# ----------------------------------------------------------------------------------------------------------

def test_block_norm_of_more_rows_than_a_launch_holds():
    """2^22 + 6 rows of 8200 columns, 1024 threads each: past 2^32 threads.  Every number is a whole one that bf16 holds."""
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 160 GiB of free memory")
    d, T = 8200, (1 << 21) + 3
    value = (torch.arange(2 * T, device="cuda") % 241).to(BF).view(2, T, 1)
    x, f = torch.empty((2, T, d), dtype=BF, device="cuda"), torch.ones((2, T, d), dtype=BF, device="cuda")
    x.copy_(value.expand_as(x))
    gate = (torch.arange(2 * d, device="cuda").view(2, d) % 13).float()
    rm.rm_block_norm(x, f, x, None, gate=gate)
    torch.cuda.synchronize()
    step = 1 << 17
    for b in range(2):
        for t in range(0, T, step):
            want = value[b, t:t + step] + gate[b].to(BF)
            assert torch.equal(x[b, t:t + step], want), (b, t)
    del x, f, want
    torch.cuda.empty_cache()


# ----------------------------------------------------------------------------------------------------------
# Bias by distance
# ----------------------------------------------------------------------------------------------------------

def biased_error(D):
    """A key's exponent is its score and slope times its distance, less that of the key where the weights lie.  Of keys with a
    weight these differ by no more than the scores do and the 40 powers of two below which weights do not count, and the slope in
    powers of two, their difference and their sum are rounded once each: 4 roundings of the score's size and 60, whatever
    the distances.  (At the least slope used, 0.07, that is 0.1 powers of two a key, 500 keys are in reach.)"""
    return lambda big: (D + 8) * U32 * big + 4 * U32 * (big + 60.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 100000), (256, 0)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_negative_slopes_on_long_caches(dtype, D, window, cap):
    """A bias that rises with the distance puts the weight on the first keys, 140 thousand from the last."""
    g = gen(42, D, window)
    N, Hq, Hk, page, length = 2, 4, 1, 64, 140000
    k, v, table = cache(g, N, -(-length // page), page, Hk, D, dtype)
    q, pos = randn(g, (N, Hq, D), dtype), ints([length - 1, length - 20000])
    slopes = torch.tensor([-0.5, -0.07, 0.5, -3.0], device="cuda")
    out = run_paged(q, k, v, table, pos, window=window, slopes=slopes, cap=cap)
    paged_within(out, q, k, v, table, pos, lambda big: biased_error(D)(big) + 16 * U32 * (big if cap else 0.0), 2.0 ** -10,
                 window=window, slopes=slopes, cap=cap, counted=1000)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("slope", [-0.5, 0.5])
def test_bias_where_the_nearest_pages_are_none(dtype, slope):
    """The weight lies far from both ends of what a token might see: the pages up to there, or from there on, are none."""
    g = gen(43, slope > 0)
    N, Hq, Hk, D, page, per = 2, 4, 2, 64, 64, 3000
    k, v, _ = cache(g, 1, 40, page, Hk, D, dtype)
    table = torch.full((N, per), -1, dtype=torch.int32)
    table[:, 1500:1520] = torch.randperm(40, generator=g).view(2, 20).to(torch.int32)
    table, q, pos = table.cuda(), randn(g, (N, Hq, D), dtype), ints([per * page - 1, per * page - 777])
    slopes = torch.full((Hq,), slope, device="cuda")
    out = run_paged(q, k, v, table, pos, slopes=slopes)
    paged_within(out, q, k, v, table, pos, biased_error(D), 2.0 ** -10, slopes=slopes, counted=1000)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("slope,D", [(0.5, 64), (-0.5, 128), (0.07, 256), (12.0, 64)])
def test_bias_on_both_sides_of_missing_pages(dtype, slope, D):
    """The first pages and the last ones are kept, those between are none: the running maximum of one side says nothing of the
    other."""
    g = gen(49, D, slope > 0)
    N, Hq, Hk, page, per = 2, 4, 2, 64, 3000
    k, v, _ = cache(g, 1, 40, page, Hk, D, dtype)
    table = torch.full((N, per), -1, dtype=torch.int32)
    kept = torch.randperm(40, generator=g).view(2, 20).to(torch.int32)
    table[:, :3], table[:, 1400], table[:, per - 9:] = kept[:, :3], kept[:, 3], kept[:, 4:13]
    table, q, pos = table.cuda(), randn(g, (N, Hq, D), dtype), ints([per * page - 1, per * page - 77])
    slopes = torch.full((Hq,), slope, device="cuda")
    out = run_paged(q, k, v, table, pos, slopes=slopes)
    paged_within(out, q, k, v, table, pos, biased_error(D), 2.0 ** -10, slopes=slopes, counted=1000)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("reach", [1.0, 0.05])
def test_one_wave_on_both_sides_of_missing_pages(dtype, reach):
    """So many heads that a wave has all keys of its head, from the first pages over the gap to the last few keys, one tile."""
    g = gen(50, int(reach * 100))
    H, D, page, per = 600, 8, 64, 3000
    k, v, _ = cache(g, 1, 20, page, H, D, dtype)
    table = torch.full((2, per), -1, dtype=torch.int32)
    table[:, :3], table[:, 1400], table[:, per - 1] = torch.arange(3), 3, torch.arange(4, 6)
    table, q, pos = table.cuda(), randn(g, (2, H, D), dtype), ints([per * page - 40, per * page - 61])
    assert rm.paged_attention_workspace(q, k, table).numel() == 0  # no head is divided
    slopes = (reach * torch.tensor([0.5, -0.5, 0.31, -4.0, 12.0, 1.7])).repeat(100).cuda()
    out = run_paged(q, k, v, table, pos, slopes=slopes)
    paged_within(out, q, k, v, table, pos, biased_error(D), 2.0 ** -10, slopes=slopes, heads=list(range(12)), counted=1000)


def test_negative_slopes_past_2_24_keys():
    """Distances that float32 does not hold, on a table that names a few pages over and over."""
    g = gen(44)
    Hq, Hk, D, page, per = 2, 1, 8, 256, 1 << 18
    k, v, _ = cache(g, 1, 37, page, Hk, D, F32)
    table = torch.randint(0, 37, (1, per), generator=g).to(torch.int32).cuda()
    q, slopes = randn(g, (1, Hq, D), F32), torch.tensor([-0.5, -0.25], device="cuda")
    out = run_paged(q, k, v, table, ints([per * page - 2]), slopes=slopes)
    # (From the thousandth key on, scores of about 3 are lowered by 250 and more.)
    paged_within(out, q, k, v, table, ints([999]), biased_error(D), 2.0 ** -10, slopes=slopes)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 256])
def test_slopes_that_leave_one_key(dtype, D):
    """Slopes so large that slope times distance passes float32: the nearest key's value, or the farthest one's."""
    g = gen(45, D)
    page = 16
    k, v, table = cache(g, 3, 300, page, 1, D, dtype)
    q, pos = randn(g, (3, 4, D), dtype), ints([0, 40, 4700])
    out = run_paged(q, k, v, table, pos, slopes=torch.tensor([1e38, -1e38, 1e30, -1e30], device="cuda"))
    for n, p in enumerate(pos.tolist()):
        near, far = v[table[n, p // page].item(), p % page, 0], v[table[n, 0].item(), 0, 0]
        for h, want in enumerate((near, far, near, far)):
            assert torch.equal(out[n, h], want), (n, h)


# ----------------------------------------------------------------------------------------------------------
# Caps
# ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap", [0.5, 5.0, 30.0, 256.0, 257.0, 1e4, 1e6, 1e8, 1e30])
@pytest.mark.parametrize("bias,window", [(False, 0), (True, 77)])
def test_caps_of_every_size(dtype, D, cap, bias, window):
    """A capped score is off by 16 roundings of its own value (the polynomial or the exponential 7, the product with the cap and
    the score over the cap one each; float32's tanhf 5), whatever the cap: no term of the cap's size."""
    g = gen(46, D, int(min(cap, 1e9)), bias)
    N, Hq, Hk, page, per = 5, 6, 2, 16, 20
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    q, pos = randn(g, (N, Hq, D), dtype), ints([3, 60, 100, 300, 319])
    slopes = torch.tensor([0.5, 0.1, 0.0, 0.03, -0.01, 0.2], device="cuda") if bias else None
    out = run_paged(q, k, v, table, pos, window=window, slopes=slopes, cap=cap)

    def error(big):
        e = biased_error(D)(big) if bias else (D + 8) * U32 * big
        return e + 16 * U32 * np.minimum(cap, big)

    paged_within(out, q, k, v, table, pos, error, 2.0 ** -10, window=window, slopes=slopes, cap=cap)


# ----------------------------------------------------------------------------------------------------------
# Batches of more tokens than a wave looks through at once (512)
# ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N", [511, 512, 513, 1024, 1025, 1300, 2049])
@pytest.mark.parametrize("D,Hq,Hk", [(64, 4, 1), (128, 8, 4), (72, 6, 6)])
@pytest.mark.parametrize("numbered", [False, True])
def test_long_batches(dtype, N, D, Hq, Hk, numbered):
    """Shares of a group that begin in every block of 512 tokens, tokens that see nothing on both sides of their borders, more
    tokens than groups and fewer."""
    g = gen(47, N, D, numbered)
    page, per = 8, 14
    k, v, table = cache(g, N, per, page, Hk, D, dtype)
    pos = (torch.rand((N,), generator=g) ** 2 * per * page).to(torch.int32)
    pos[::11] = -1
    for border in range(512, N + 1, 512):
        pos[border - 9:border + 14] = -3
        pos[border - 2:border] = per * page - 1
    pos[N - 1] = 77
    seq = torch.randperm(N, generator=g).to(torch.int32).cuda() if numbered else None
    q, pos = randn(g, (N, Hq, D), dtype), pos.cuda()
    out = run_paged(q, k, v, table, pos, seq=seq)
    paged_within(out, q, k, v, table, pos, lambda big: (D + 8) * U32 * big, 2.0 ** -10, seq=seq, heads=[0, Hq - 1])
    assert (out[pos < 0] == 0).all() and out.isfinite().all()


@pytest.mark.parametrize("N", [600, 1500])
def test_long_batches_with_one_long_cache(N):
    """The keys of nearly all groups are one token's, in the first, the second and the last block."""
    g = gen(48, N)
    D, page, per, Hq, Hk = 64, 16, 600, 4, 2
    k, v, _ = cache(g, 1, per, page, Hk, D, BF)
    table = torch.stack([torch.randperm(per, generator=g) for _ in range(4)]).to(torch.int32).cuda()
    seq = torch.randint(0, 4, (N,), generator=g).to(torch.int32).cuda()
    for at in (3, 513, N - 1):
        pos = (torch.rand((N,), generator=g) * 20).to(torch.int32) - 2
        pos[at] = per * page - 1
        q, pos = randn(g, (N, Hq, D), BF), pos.cuda()
        out = run_paged(q, k, v, table, pos, seq=seq)
        paged_within(out, q, k, v, table, pos, lambda big: (D + 8) * U32 * big, 2.0 ** -10, seq=seq, heads=[0, 3])
