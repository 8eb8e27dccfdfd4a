"""GPU tests of the serving-step calls where their bounds are tight: weights of bf16 attention to 2^-15.

Bound (u32 = 2^-24, u = the output type's half step): as in test_gpu_serving.py, with the weights in two bf16 parts: the
first by truncation, which leaves a rest below 2^-7 of the weight, the second the rest rounded by at most 2^-8 of it, so a
weight is off by 2^-15.  A bound is worth its name while it leaves little beside the output's own rounding: of every case the
rest is at most `spare` of the softmax average of |v|."""
import numpy as np
import pytest
import torch

import paper_2609_19104_amd as rm
from oracle import serving

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_serving import BF, F32, U, U32, cache, f64, gen, ints, randn, run_paged  # noqa: E402


def paged_within(out, q, k, v, table, pos, e, spare, seq=None, window=0, slopes=None, scale=None, cap=0.0, heads=None):
    """out against the oracle, e(big) the bound of a score's error, big the score's size sum |q||k| scale."""
    D = q.shape[2]
    s = np.float32(D ** -0.5 if scale is None else scale)
    ref, mag, big = serving.paged_attention(f64(q), f64(k), f64(v), table.cpu().numpy(),
                                            None if seq is None else seq.cpu().numpy(), pos.cpu().numpy(), window, s, cap,
                                            f64(slopes), heads)
    longest = min(int(pos.max()) + 1, table.shape[1] * k.shape[1])
    x = e(big[..., None])
    rest = 2 * x * (1 + x) + (2.0 ** -15 if q.dtype == BF else 0.0) + (longest + 32) * U32
    got, at = f64(out), slice(None) if heads is None else heads
    assert rest[:, at].max() <= spare
    tol = (U[q.dtype] * np.abs(ref) + (1 + U[q.dtype]) * rest * mag + 1e-30)[:, at]
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
