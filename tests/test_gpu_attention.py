"""GPU tests of rm_span_attention, rm_prefix_attention, rm_attn_spans and rm_qk_norm_rope against the float64 oracle.

Bounds (u32 = 2^-24 the unit roundoff of float32, u = that of the output type):
  attention: |o - ref| <= u |ref| + (2 e + uP + (N + 32) u32) mag, with mag the softmax average of |v|, uP = 2^-8 the
             rounding of the weights in bf16 (0 in float32), and e a bound on a score's absolute error: the product's
             D + 4 roundings of scale sum |q||k|, three roundings of the score, of the bias and of its log2 e form, and
             with a cap c the tanh's, of which 1 - 2 / (1 + e^2x) has at most 6 roundings of values up to c (2 c covers
             the reciprocal's and exp2's last places).  A weight e^s is then off by at most e (1 + e) relatively, the
             sum of the weights too, hence 2 e.
  rotation:  |y - ref| <= u |ref| + r ((D / 2 + 16) u32 + 8 u32 + 5 2^-53 |pos f|), r the length of the element's pair
             (at least the element): the sum of squares, the factor and gain, the products, the sine and cosine, and the
             angle, whose turns are formed in float64."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as att

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_19104_amd as rm  # noqa: E402

U32 = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
BF, F32 = torch.bfloat16, torch.float32


def gen(*path):
    g = torch.Generator()
    s = 17
    for p in path:
        s = s * 1000003 + int(p)
    g.manual_seed(s % (1 << 62))
    return g


def randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def bound(ref, mag, big, dtype, D, n, cap=0.0, bias=0.0):
    e = (D + 8) * U32 * big[..., None] + 4 * U32 * bias + (16 * U32 * cap if cap else 0.0)
    up = 2.0 ** -8 if dtype == BF else 0.0
    return U[dtype] * np.abs(ref) + (2 * e * (1 + e) + up + (n + 32) * U32) * mag + 1e-30


def check(out, ref, tol):
    got = f64(out)
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    worst = float(np.max(err / np.maximum(tol, 1e-30))) if err.size else 0.0
    assert worst <= 1.0, f"error {worst:.3f} times the bound (largest {err.max():.3e})"


def run_span(q, k, v, span=None, slopes=None, q_start=None, scale=None, cap=0.0):
    out = torch.full_like(q, float("nan"))
    ws = rm.span_attention_workspace(q, k)
    ws.fill_(0xFF)
    rm.rm_span_attention(q, k, v, out, ws, span=span, slopes=slopes, q_start=q_start, scale=scale, softcap=cap)
    torch.cuda.synchronize()
    return out


def check_span(q, k, v, span=None, slopes=None, q_start=None, scale=None, cap=0.0, out=None):
    B, T, Hq, D = q.shape
    N = k.shape[1]
    if out is None:
        out = run_span(q, k, v, span, slopes, q_start, scale, cap)
    sp = np.broadcast_to(np.array([0, N]), (B, T, 2)) if span is None else np.clip(span.cpu().numpy(), 0, N)
    s = D ** -0.5 if scale is None else scale
    ref, mag, big = att.span_attention(f64(q), f64(k), f64(v), sp, np.float32(s), cap,
                                       None if slopes is None else f64(slopes),
                                       None if q_start is None else q_start.cpu().numpy())
    bias = 0.0
    if slopes is not None:
        far = max(N, T) + (0 if q_start is None else int(q_start.abs().max()))
        bias = float(slopes.abs().max()) * far
    check(out, ref, bound(ref, mag, big, q.dtype, D, N, cap, bias))
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 64, 72, 128, 200, 256])
@pytest.mark.parametrize("T,N", [(1, 1), (5, 33), (40, 129)])
def test_full_spans(dtype, D, T, N):
    g = gen(1, D, T, N)
    check_span(randn(g, (2, T, 4, D), dtype, 2.0), randn(g, (2, N, 2, D), dtype), randn(g, (2, N, 2, D), dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", list(range(16, 257, 24)) + [96, 192])
@pytest.mark.parametrize("many", [False, True])
def test_every_kernel_width(dtype, D, many):
    """Head widths inside each of the kernels' classes, with keys whose infinite components a row sees: a score of
    -infinity has no weight, +infinity none that is defined."""
    g = gen(11, D, many)
    B, T, N, Hq, Hk = (40, 130, 130, 16, 16) if many else (2, 12, 140, 4, 2)
    q, k, v = randn(g, (B, T, Hq, D), dtype, 2.0), randn(g, (B, N, Hk, D), dtype), randn(g, (B, N, Hk, D), dtype)
    q[..., D - 1] = q[..., D - 1].abs() + 0.5
    out = run_span(q, k, v)
    for b, h in ((0, 0), (B - 1, Hq - 1)):
        kv = h // (Hq // Hk)
        check_span(q[b:b + 1, :, h:h + 1], k[b:b + 1, :, kv:kv + 1], v[b:b + 1, :, kv:kv + 1], out=out[b:b + 1, :, h:h + 1])
    span = torch.tensor([1, N], dtype=torch.int32, device="cuda").expand(B, T, 2).contiguous()
    k2 = k.clone()
    k2[:, 0, :, D - 1] = -float("inf")
    out = run_span(q, k2, v)
    for b, h in ((0, 0), (B - 1, Hq - 1)):  # as if the first key were not there
        kv = h // (Hq // Hk)
        check_span(q[b:b + 1, :, h:h + 1], k[b:b + 1, :, kv:kv + 1], v[b:b + 1, :, kv:kv + 1], span[b:b + 1],
                   out=out[b:b + 1, :, h:h + 1])
    k[:, 0, :, D - 1] = float("inf")
    assert bool(run_span(q, k, v).isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (8, 1), (6, 2), (40, 1)])
def test_head_layouts(dtype, Hq, Hk):
    g = gen(2, Hq, Hk)
    check_span(randn(g, (1, 9, Hq, 64), dtype, 2.0), randn(g, (1, 70, Hk, 64), dtype), randn(g, (1, 70, Hk, 64), dtype))


def random_spans(g, B, T, N):
    a = torch.randint(-5, N + 6, (B, T, 2), generator=g, dtype=torch.int32)
    a[:, ::7] = 0           # rows that see nothing
    return a.cuda()         # and ends out of order or outside [0, N], which see nothing or are cut


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_random_spans_cap_and_bias(dtype, D, cap, bias):
    g = gen(3, D, int(cap), bias)
    B, T, N, Hq, Hk = 2, 45, 201, 4, 2
    slopes = torch.tensor([0.5, 0.1, 0.0, 0.03], device="cuda") if bias else None
    start = ints([13, -4]) if bias else None
    check_span(randn(g, (B, T, Hq, D), dtype, 2.0), randn(g, (B, N, Hk, D), dtype), randn(g, (B, N, Hk, D), dtype),
               random_spans(g, B, T, N), slopes, start, 0.11, cap)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_rows(dtype, D):
    """Enough row blocks for the kernel whose waves divide the rows: causal spans and random ones."""
    g = gen(4, D)
    B, T, N, H = 33, 130, 130, 16
    q, k, v = (randn(g, (B, T, H, D), dtype, s) for s in (2.0, 1.0, 1.0))
    span = torch.empty((B, T, 2), dtype=torch.int32, device="cuda")
    rm.rm_attn_spans(span, N, causal=True)
    span[1] = random_spans(g, 1, T, N)[0]
    out = run_span(q, k, v, span)
    for b in (0, 1, B - 1):
        for h in (0, H - 1):
            cut = [t[b:b + 1, :, h:h + 1] for t in (q, k, v, out)]
            check_span(*cut[:3], span[b:b + 1], out=cut[3])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,Hq,Hk", [(64, 8, 1), (128, 4, 2), (256, 8, 1), (72, 2, 2)])
@pytest.mark.parametrize("T,N", [(1, 3001), (3, 5000)])
def test_long_keys_and_few_rows(dtype, D, Hq, Hk, T, N):
    """Several workgroups divide the keys; one sample sees few of them, so that some get none."""
    g = gen(5, D, T)
    q, k, v = randn(g, (2, T, Hq, D), dtype, 2.0), randn(g, (2, N, Hk, D), dtype), randn(g, (2, N, Hk, D), dtype)
    span = torch.empty((2, T, 2), dtype=torch.int32, device="cuda")
    rm.rm_attn_spans(span, N, causal=True, q_start=ints([N - T, 100]))
    assert rm.span_attention_workspace(q, k).numel() > 0
    check_span(q, k, v, span, slopes=torch.linspace(0.001, 0.1, Hq, device="cuda"), q_start=ints([N - T, 100]))
    check_span(q, k, v, span, cap=30.0)
    span.zero_()
    assert not run_span(q, k, v, span).any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_keys_and_one_key(dtype):
    g = gen(6)
    q = randn(g, (2, 3, 4, 64), dtype)
    e = torch.empty((2, 0, 2, 64), dtype=dtype, device="cuda")
    assert not run_span(q, e, e).any()
    k, v = randn(g, (2, 1, 2, 64), dtype), randn(g, (2, 1, 2, 64), dtype)
    assert torch.equal(run_span(q, k, v), v.repeat_interleave(2, 2).expand(2, 3, 4, 64))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides(dtype):
    """Views of one projection's rows, head-major tensors, one head's keys for all, and rows around the output kept."""
    g = gen(7)
    B, T, Hq, Hk, D = 2, 37, 6, 2, 64
    qkv = randn(g, (B, T, Hq + 2 * Hk, D), dtype)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    ref = check_span(q, k, v)
    assert torch.equal(run_span(q.contiguous(), k.contiguous(), v.contiguous()), ref)
    hm = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v)]
    big = torch.full((B, Hq, T + 5, D + 16), 7.0, dtype=dtype, device="cuda")
    out = big[:, :, 2:2 + T, 8:8 + D].permute(0, 2, 1, 3)
    rm.rm_span_attention(*hm, out, rm.span_attention_workspace(hm[0], hm[1]))
    assert torch.equal(out, ref)
    out.fill_(7.0)
    assert bool((big == 7.0).all())
    one = k[:, :, :1].expand(B, T, Hk, D)
    assert torch.equal(run_span(q, one, one), run_span(q, one.contiguous(), one.contiguous()))
    same = k[:1].expand(B, T, Hk, D)
    assert torch.equal(run_span(q, same, same), run_span(q, same.contiguous(), same.contiguous()))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("many", [False, True])
def test_unseen_keys_may_hold_anything(dtype, D, many):
    """NaN and infinities in keys and values that a row does not see leave it bit for bit, also where rows of the same
    tile see them; the rows that do get what the definition gives."""
    g = gen(8, D)
    B, T, N, Hq, Hk = (40, 130, 130, 16, 16) if many else (2, 20, 150, 4, 2)
    q, k, v = randn(g, (B, T, Hq, D), dtype, 2.0), randn(g, (B, N, Hk, D), dtype), randn(g, (B, N, Hk, D), dtype)
    span = torch.empty((B, T, 2), dtype=torch.int32, device="cuda")
    rm.rm_attn_spans(span, N, causal=True, kv_len=torch.full((B,), N - 9, dtype=torch.int32, device="cuda"))
    want = run_span(q, k, v, span)
    bad = T // 2
    k2, v2 = k.clone(), v.clone()
    k2[:, N - 9:] = float("nan")
    v2[:, N - 9:] = float("inf")
    assert torch.equal(run_span(q, k2, v2, span), want)
    v2[:, bad, :, 0] = float("nan")
    v2[:, bad, :, 1] = float("inf")
    v2[:, bad, :, 2] = -float("inf")
    v2[:, bad, :, D - 1] = -float("inf")
    got = run_span(q, k2, v2, span)
    assert torch.equal(got[:, :bad], want[:, :bad])
    end = min(T, N - 9)  # rows from kv_len on see nothing
    rest = got[:, bad:end]
    assert not got[:, end:].any()
    assert bool(rest[..., 0].isnan().all()) and bool((rest[..., 1] == float("inf")).all())
    assert bool((rest[..., 2] == -float("inf")).all()) and bool((rest[..., D - 1] == -float("inf")).all())
    keep = torch.ones(D, dtype=torch.bool, device="cuda")
    keep[[0, 1, 2, D - 1]] = False
    assert torch.equal(rest[..., keep], want[:, bad:end][..., keep])
    k2[:, bad] = float("nan")
    got = run_span(q, k2, v, span)
    assert torch.equal(got[:, :bad], want[:, :bad]) and bool(got[:, bad:end].isnan().all())


def test_large_scores():
    """Scores in the thousands, rising and falling along the keys: the running maximum's rescaling."""
    for dtype in (BF, F32):
        N, D = 400, 64
        q = torch.zeros((1, 2, 1, D), dtype=dtype, device="cuda")
        q[0, 0, 0, 0], q[0, 1, 0, 0] = 8.0, -8.0
        k = torch.zeros((1, N, 1, D), dtype=dtype, device="cuda")
        k[0, :, 0, 0] = torch.arange(N, device="cuda").to(dtype)
        v = randn(gen(9), (1, N, 1, D), dtype)
        check_span(q, k, v, scale=1.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,many", [(8, False), (64, False), (72, False), (128, False), (200, False),
                                    (256, False), (64, True), (128, True), (256, True)])
@pytest.mark.parametrize("cap", [256.0, 257.0, 1e4, 1e6, 1e8, 1e30])
@pytest.mark.parametrize("bias", [False, True])
def test_high_caps(dtype, D, many, cap, bias):
    """Caps far above the scores leave these as they are: from 256 on the tanh is off by 16 roundings of its value (the
    polynomial 7, the product with the cap and the score over the cap one each; float32's tanhf 5), so the bound's e has
    16 u32 of the score and no term of the cap's size.  At 256 itself such a term is 16 u32 256 = 0.00024."""
    g = gen(14, D, many, bias)
    B, T, N, Hq, Hk = (40, 130, 130, 16, 16) if many else (2, 12, 300, 4, 2)
    q, k, v = randn(g, (B, T, Hq, D), dtype, 2.0), randn(g, (B, N, Hk, D), dtype), randn(g, (B, N, Hk, D), dtype)
    slopes = torch.linspace(0.01, 0.1, Hq, device="cuda") if bias else None
    out = run_span(q, k, v, slopes=slopes, cap=cap)
    for b, h in ((0, 0), (B - 1, Hq - 1)):
        kv = h // (Hq // Hk)
        one = None if slopes is None else f64(slopes)[h:h + 1]
        cut = [f64(t) for t in (q[b:b + 1, :, h:h + 1], k[b:b + 1, :, kv:kv + 1], v[b:b + 1, :, kv:kv + 1])]
        span = np.broadcast_to(np.array([0, N]), (1, T, 2))
        ref, mag, big = att.span_attention(*cut, span, np.float32(D ** -0.5), cap, one)
        tol = bound(ref, mag, big, dtype, D + 16, N, cap if cap == 256.0 else 0.0, 0.0 if one is None else float(one[0]) * N)
        check(out[b:b + 1, :, h:h + 1], ref, tol)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,T,N", [(64, 5, 300), (128, 40, 150), (256, 3, 4000)])
@pytest.mark.parametrize("start", [-(1 << 31), -(1 << 30) - 3, -100000001, 100000001, (1 << 30) + 7, (1 << 31) - 2])
def test_positions_far_from_the_keys(dtype, D, T, N, start):
    """Every key is on one side of such a row, so its distances are those from that end but for a constant that the
    softmax does not see: their error is that of distances up to N."""
    g = gen(15, D, T, start & 0xffffffff)
    Hq, Hk = 4, 2
    q, k, v = randn(g, (2, T, Hq, D), dtype, 2.0), randn(g, (2, N, Hk, D), dtype), randn(g, (2, N, Hk, D), dtype)
    slopes = torch.tensor([0.25, 0.1, 0.0, 0.03], device="cuda")
    starts = ints([start, N - T])
    out = run_span(q, k, v, None, slopes, starts)
    span = np.broadcast_to(np.array([0, N]), (2, T, 2))
    ref, mag, big = att.span_attention(f64(q), f64(k), f64(v), span, np.float32(D ** -0.5), 0.0, f64(slopes),
                                       starts.cpu().numpy().astype(np.int64))
    check(out, ref, bound(ref, mag, big, dtype, D, N, 0.0, 0.25 * (N + T)))


def test_offsets_past_32_bits():
    D, Hk, N = 128, 8, 4096
    big = torch.zeros((300, N, Hk, D), dtype=BF, device="cuda")  # 2.5 GB a tensor, in elements past 2^31
    g = gen(10)
    q, k, v = randn(g, (1, 2, 8, D), BF), randn(g, (1, N, Hk, D), BF), randn(g, (1, N, Hk, D), BF)
    big[299], big[298] = k[0], v[0]
    base = run_span(q, k, v)
    out = torch.empty((300, 2, 8, D), dtype=BF, device="cuda")
    rm.rm_span_attention(q.expand(300, 2, 8, D), big, big[298:299].expand(300, N, Hk, D), out,
                         rm.span_attention_workspace(out, big))
    assert torch.allclose(out[299].float(), base[0].float(), atol=2e-2, rtol=2e-2)
    far = big.view(1, 300 * N, Hk, D)  # one sample of 1.2 million keys: byte offsets to 2.5 GB
    span = torch.tensor([[[299 * N, 300 * N]] * 2], dtype=torch.int32, device="cuda")
    vv = torch.zeros_like(far)
    vv[0, 299 * N:] = v[0]
    assert torch.allclose(run_span(q, far, vv, span).float(), base.float(), atol=2e-2, rtol=2e-2)


def test_widest_token_stride():
    """Tokens just below 16 MiB apart: a tile's offsets pass 2^31 bytes."""
    D, N, step = 64, 130, (1 << 23) - 8
    buf = torch.zeros((N * step,), dtype=BF, device="cuda")
    g = gen(12)
    k, v = (torch.as_strided(buf, (1, N, 2, D), (0, step, 128, 1), at) for at in (0, 512))
    k.copy_(randn(g, (1, N, 2, D), BF))
    v.copy_(randn(g, (1, N, 2, D), BF))
    q = randn(g, (1, 3, 4, D), BF)
    out = check_span(q, k, v)
    assert torch.equal(run_span(q, k.contiguous(), v.contiguous()), out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,Hk,T", [(35, 5, 13), (9, 3, 50), (11, 1, 3), (64, 1, 5)])
def test_heads_that_do_not_divide_the_row_blocks(dtype, Hq, Hk, T):
    g = gen(13, Hq, T)
    N = 77
    check_span(randn(g, (3, T, Hq, 64), dtype, 2.0), randn(g, (3, N, Hk, 64), dtype), randn(g, (3, N, Hk, 64), dtype),
               random_spans(g, 3, T, N), torch.linspace(0, 0.2, Hq, device="cuda"), ints([5, 0, 70]))


# ---------------------------------------------------------------------------------------------- shared prefix

def run_prefix(q, kp, vp, ko, vo, plen=None, olen=None, causal=False, scale=None, cap=0.0):
    out = torch.full_like(q, float("nan"))
    ws = rm.prefix_attention_workspace(q, kp, ko)
    ws.fill_(0xFF)
    rm.rm_prefix_attention(q, kp, vp, ko, vo, out, ws, prefix_len=plen, own_len=olen, causal=causal, scale=scale,
                           softcap=cap)
    torch.cuda.synchronize()
    return out


def make_prefix(g, G, per, T, P, S, Hq, Hk, D, dtype):
    return (randn(g, (G * per, T, Hq, D), dtype, 2.0), randn(g, (G, P, Hk, D), dtype), randn(g, (G, P, Hk, D), dtype),
            randn(g, (G * per, S, Hk, D), dtype), randn(g, (G * per, S, Hk, D), dtype))


def check_prefix(args, plen=None, olen=None, causal=False, cap=0.0):
    out = run_prefix(*args, plen, olen, causal, None, cap)
    D = args[0].shape[-1]
    ref, mag, big = att.prefix_attention(*(f64(a) for a in args), np.float32(D ** -0.5), cap,
                                         None if plen is None else plen.cpu().numpy(),
                                         None if olen is None else olen.cpu().numpy(), causal)
    check(out, ref, bound(ref, mag, big, args[0].dtype, D, args[1].shape[1] + args[3].shape[1], cap))
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,per,T,P,S,Hq,Hk,D", [
    (1, 1, 1, 1, 1, 1, 1, 64), (1, 3, 5, 70, 9, 4, 2, 64), (2, 5, 1, 130, 20, 8, 2, 128), (2, 2, 11, 50, 11, 8, 1, 256),
    (3, 40, 1, 33, 6, 2, 1, 72), (1, 4, 3, 0, 7, 2, 2, 128), (2, 3, 2, 65, 0, 4, 1, 64), (1, 2, 2, 0, 0, 2, 1, 64),
    (1, 70, 33, 90, 33, 8, 8, 64),
])
def test_prefix(dtype, G, per, T, P, S, Hq, Hk, D):
    g = gen(20, per, T, P, S, D)
    check_prefix(make_prefix(g, G, per, T, P, S, Hq, Hk, D, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("T,D", [(1, 64), (4, 128), (30, 256)])
def test_prefix_ragged(dtype, causal, cap, T, D):
    g = gen(21, T, D, causal)
    G, per, P, S, Hq, Hk = 2, 6, 150, 45, 4, 2
    args = make_prefix(g, G, per, T, P, S, Hq, Hk, D, dtype)
    olen = ints([45, 0, 1, 3, 17, 33, 44, 32, 100, -4, 2, 31])  # lengths outside [0, S] are cut
    out = check_prefix(args, ints([0, 131]), olen, causal, cap)
    assert not out[1].any()  # no prefix and no own key
    check_prefix(args, ints([1000, -1]), olen, causal, cap)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prefix_long_and_few_rows(dtype, D):
    g = gen(22, D)
    args = make_prefix(g, 1, 3, 1, 4000, 700, 8, 2, D, dtype)
    assert rm.prefix_attention_workspace(args[0], args[1], args[3]).numel() > 0
    check_prefix(args, ints([3777]), ints([700, 3, 0]), True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("P", [70, 400])
def test_prefix_many_rows(dtype, D, causal, P):
    """Many rows, each wave with samples of its own, on many own keys (waves that divide the keys) and on a longer
    prefix (waves that divide the rows); two samples hold NaN."""
    g = gen(24, D)
    G, per, T, S, H = 2, 75, 33, 40, 16
    q, kp, vp, ko, vo = make_prefix(g, G, per, T, P, S, H, H, D, dtype)
    olen = torch.randint(0, S + 1, (G * per,), generator=g, dtype=torch.int32)
    olen[0], olen[1], olen[-1] = S, 0, 1
    plen = ints([P, 33])
    ko[5], vo[80] = float("nan"), float("nan")
    out = run_prefix(q, kp, vp, ko, vo, plen, olen.cuda(), causal)
    for b in (0, 1, 2, 4, 6, 74, 75, 79, 81, 149):
        i = b // per
        for h in (0, H - 1):
            a = [t[:, :, h:h + 1] for t in (q[b:b + 1], kp[i:i + 1], vp[i:i + 1], ko[b:b + 1], vo[b:b + 1])]
            ref, mag, big = att.prefix_attention(*(f64(t) for t in a), np.float32(D ** -0.5), 0.0, [int(plen[i])],
                                                 [int(olen[b])], causal)
            check(out[b:b + 1, :, h:h + 1], ref, bound(ref, mag, big, dtype, D, P + S))


@pytest.mark.parametrize("D,per", [(64, 24), (128, 24), (256, 16)])
@pytest.mark.parametrize("causal", [False, True])
def test_row_waves_and_slices(D, per, causal):
    """Blocks of 128 rows whose keys two workgroups divide, of a shared prefix and of spans."""
    g = gen(25, D)
    G, T, P, S, Hq = 2, 32, 4000, 60, 16
    q, kp, vp, ko, vo = make_prefix(g, G, per, T, P, S, Hq, 1, D, BF)
    assert rm.prefix_attention_workspace(q, kp, ko).numel() > 0
    olen = torch.randint(0, S + 1, (G * per,), generator=g, dtype=torch.int32)
    olen[0], olen[-1] = S, 0
    plen = ints([P, 77])
    out = run_prefix(q, kp, vp, ko, vo, plen, olen.cuda(), causal)
    assert torch.equal(out, run_prefix(q, kp, vp, ko, vo, plen, olen.cuda(), causal))
    for b in (0, 1, per - 1, per, G * per - 1):
        i = b // per
        a = [t for t in (q[b:b + 1, :, 3:5], kp[i:i + 1], vp[i:i + 1], ko[b:b + 1], vo[b:b + 1])]
        ref, mag, big = att.prefix_attention(*(f64(t) for t in a), np.float32(D ** -0.5), 0.0, [int(plen[i])],
                                             [int(olen[b])], causal)
        check(out[b:b + 1, :, 3:5], ref, bound(ref, mag, big, BF, D, P + S))
    q = randn(g, (4, 32 * per // 24 * 24, Hq * 2, D), BF, 2.0)
    span = torch.empty((4, q.shape[1], 2), dtype=torch.int32, device="cuda")
    k, v = randn(g, (4, P, 1, D), BF), randn(g, (4, P, 1, D), BF)
    rm.rm_attn_spans(span, P, causal=causal, q_start=ints([0, 100, P - 500, 7]))
    out = run_span(q, k, v, span)
    for b, h in ((0, 0), (2, 31)):
        check_span(q[b:b + 1, ::37, h:h + 1], k[b:b + 1], v[b:b + 1], span[b:b + 1, ::37], out=out[b:b + 1, ::37, h:h + 1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,per,T,P,S,Hq,Hk,D", [
    (1, 32, 1, 128, 256, 8, 8, 128), (1, 32, 1, 0, 300, 8, 8, 64), (2, 16, 1, 200, 512, 4, 1, 128), (1, 40, 2, 33, 400, 6, 2, 72),
    (1, 3, 51, 100, 1500, 8, 1, 256),
])
def test_slices_of_many_samples(dtype, G, per, T, P, S, Hq, Hk, D):
    """Workgroups that divide the own keys of a row block's many samples; every other sample has few, some none."""
    g = gen(28, per, T, P, S, D)
    args = make_prefix(g, G, per, T, P, S, Hq, Hk, D, dtype)
    assert rm.prefix_attention_workspace(args[0], args[1], args[3]).numel() > 0
    olen = torch.randint(0, S + 1, (G * per,), generator=g, dtype=torch.int32)
    olen[1::2] = torch.randint(0, 9, olen[1::2].shape, generator=g, dtype=torch.int32)
    check_prefix(args, None, olen.cuda(), True)
    check_prefix(args, ints([P // 2] * G), olen.cuda())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("T,B,N", [(5, 2, 70000), (12, 2, 70000), (5, 200, 130)])
def test_blocks_that_are_not_full(D, T, B, N):
    """40 and 96 rows to a key head: few blocks on many keys, many on few."""
    g = gen(27, D, T, B)
    q, k, v = randn(g, (B, T, 32, D), BF, 2.0), randn(g, (B, N, 4, D), BF), randn(g, (B, N, 4, D), BF)
    hi = torch.randint(0, N + 1, (B, T, 1), generator=g)
    span = torch.cat([torch.zeros_like(hi), hi], -1).to(torch.int32).cuda()
    out = run_span(q, k, v, span)
    for b, h in ((0, 0), (B // 2, 17), (B - 1, 31)):
        check_span(q[b:b + 1, :, h:h + 1], k[b:b + 1, :, h // 8:h // 8 + 1], v[b:b + 1, :, h // 8:h // 8 + 1],
                   span[b:b + 1], out=out[b:b + 1, :, h:h + 1])


@pytest.mark.parametrize("dtype,D,T,N", [(BF, 64, 512, 20000), (BF, 128, 512, 20000), (BF, 256, 128, 20000),
                                         (BF, 128, 512, 33000), (BF, 256, 128, 33000), (F32, 128, 40, 9000),
                                         (BF, 128, 3, 9000)])
def test_slices_that_see_no_keys(dtype, D, T, N):
    """Few rows on many keys, of which each sees few or none: most workgroups of a row block have nothing to do."""
    g = gen(26, D, T, N)
    q = randn(g, (2, T, 8, D), dtype, 2.0)
    k, v = randn(g, (2, N, 1, D), dtype), randn(g, (2, N, 1, D), dtype)
    assert rm.span_attention_workspace(q, k).numel() > 0
    lo = torch.randint(0, N, (2, 1, 1), generator=g) + torch.randint(0, 200, (2, T, 1), generator=g)
    span = torch.cat([lo, lo + torch.randint(0, 300, (2, T, 1), generator=g)], -1).clamp(max=N).to(torch.int32)
    span[1, T // 2:] = 0
    span = span.cuda()
    out = run_span(q, k, v, span)
    step = max(1, T // 9)
    for h in (0, 7):
        check_span(q[:, ::step, h:h + 1], k, v, span[:, ::step], out=out[:, ::step, h:h + 1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 20])
def test_one_samples_nan_stays_its_own(dtype, T):
    g = gen(23, T)
    q, kp, vp, ko, vo = make_prefix(g, 2, 6, T, 40, 30, 4, 1, 64, dtype)
    olen = ints([30, 29, 12, 7, 30, 1] * 2)
    want = run_prefix(q, kp, vp, ko, vo, None, olen)
    ko2, vo2 = ko.clone(), vo.clone()
    ko2[2], vo2[2], vo2[7, 3] = float("nan"), float("nan"), float("inf")
    for b in range(12):  # rows past the lengths
        vo2[b, int(olen[b]):] = float("nan")
        ko2[b, int(olen[b]):] = float("inf")
    got = run_prefix(q, kp, vp, ko2, vo2, None, olen)
    others = [b for b in range(12) if b not in (2, 7)]
    assert torch.equal(got[others], want[others])
    assert bool(got[2].isnan().all()) and bool((got[7] == float("inf")).all())


def poisoned(v, keys):
    """v with NaN, infinities or both signs of them in five columns of the listed keys ([(sample, key)]), and per column
    what a row that sees the key gets."""
    D = v.shape[-1]
    out = v.clone()
    marks = {c: torch.zeros(v.shape[:2] + (3,), dtype=torch.bool) for c in (0, 1, 2, 3, D - 1)}  # NaN, +, - of each key
    for n, (b, j) in enumerate(keys):
        for c, kind in ((0, 0), (1, 1), (2, 2), (3, 1 + n % 2), (D - 1, n % 3)):
            out[b, j, :, c] = (float("nan"), float("inf"), -float("inf"))[kind]
            marks[c][b, j, kind] = True
    return out, marks


def check_poisoned(got, want, seen, marks):
    """got, want [B][T][H][D], seen [B][T][N] on the host: columns of rows that see marked keys get their infinity or
    NaN, everything else its bits."""
    got, want = got.cpu(), want.cpu()
    for c in range(got.shape[-1]):
        if c not in marks:
            assert torch.equal(got[..., c], want[..., c]), c
            continue
        hit = torch.einsum("btn,bnk->btk", seen.float(), marks[c].float()) > 0
        nan = hit[..., 0] | (hit[..., 1] & hit[..., 2])
        kinds = ((nan, "nan"), (hit[..., 1] & ~nan, "inf"), (hit[..., 2] & ~nan, "-inf"), (~hit.any(-1), None))
        for rows, value in kinds:
            x = got[..., c][rows]
            if value is None:
                assert torch.equal(x, want[..., c][rows]), c
            else:
                assert bool(x.isnan().all() if value == "nan" else (x == float(value)).all()), (c, value)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 64, 72, 128, 136, 200, 256])
@pytest.mark.parametrize("T,N", [(20, 5000), (3, 3001), (20, 150)])
def test_unseen_values_in_slices(dtype, D, T, N):
    """Infinities and NaN among the values of a few keys of many tiles, which some rows of a block see and others not:
    in whole calls (N = 150 up to 128 columns) and in those whose keys many workgroups divide."""
    g = gen(16, D, T, N)
    B, Hq, Hk = 2, 4, 2
    q, k, v = randn(g, (B, T, Hq, D), dtype), randn(g, (B, N, Hk, D), dtype), randn(g, (B, N, Hk, D), dtype)
    lo = torch.randint(0, N, (B, T), generator=g)
    hi = lo + torch.where(torch.rand((B, T), generator=g) < 0.5, torch.randint(0, 60, (B, T), generator=g),
                          torch.randint(0, N, (B, T), generator=g))
    span = torch.stack([lo, hi.clamp(max=N)], -1).to(torch.int32)
    span[0, 1] = 0
    assert N < 1000 or rm.span_attention_workspace(q, k).numel() > 0
    j = torch.arange(N)
    seen = (j >= span[..., :1]) & (j < span[..., 1:])
    want = run_span(q, k, v, span.cuda())
    step = 131 if N > 1000 else 40
    v2, marks = poisoned(v, [(b, i) for b in range(B) for i in range(5 + 7 * b, N, step)])
    got = run_span(q, k, v2, span.cuda())
    check_poisoned(got, want, seen, marks)
    graph = torch.cuda.CUDAGraph()
    out, ws, sp = torch.empty_like(q), rm.span_attention_workspace(q, k), span.cuda()
    rm.rm_span_attention(q, k, v2, out, ws, span=sp)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rm.rm_span_attention(q, k, v2, out, ws, span=sp)
    for _ in range(3):
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16 if dtype == BF else torch.int32),
                           got.view(torch.int16 if dtype == BF else torch.int32))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 72, 128, 256])
@pytest.mark.parametrize("G,per,T,P,S,Hq,Hk", [(1, 6, 2, 3000, 400, 4, 1), (2, 5, 3, 40, 700, 8, 2), (1, 40, 1, 0, 300, 2, 1)])
def test_own_keys_infinite_values_in_slices(dtype, D, G, per, T, P, S, Hq, Hk):
    """The same among the samples' own keys and in the shared ones, with lengths that hide some of them."""
    g = gen(17, D, per, P, S)
    q, kp, vp, ko, vo = make_prefix(g, G, per, T, P, S, Hq, Hk, D, dtype)
    q = q * 0.5
    assert rm.prefix_attention_workspace(q, kp, ko).numel() > 0
    olen = torch.randint(0, S + 1, (G * per,), generator=g, dtype=torch.int32)
    olen[0], olen[1] = S, 0
    plen = torch.tensor([P - P // 3, P // 2][:G], dtype=torch.int32)
    want = run_prefix(q, kp, vp, ko, vo, plen.cuda(), olen.cuda(), True)
    own_bad = [(b, i) for b in range(0, G * per, 2) for i in range(3 + b % 5, S, 77)]
    vo2, marks = poisoned(vo, own_bad)
    j = torch.arange(S)
    seen = (j < olen[:, None, None]) & (j <= (olen[:, None, None] - T + torch.arange(T)[:, None]))
    check_poisoned(run_prefix(q, kp, vp, ko, vo2, plen.cuda(), olen.cuda(), True), want, seen, marks)
    if P > 0:
        vp2, marks = poisoned(vp, [(u, i) for u in range(G) for i in range(int(plen[u]) - 200 * (u + G - 2), P, 150)
                                   if i >= 0])
        sees = (torch.arange(P) < plen[:, None]).repeat_interleave(per, 0)[:, None].expand(G * per, T, P)
        marks = {c: m.repeat_interleave(per, 0) for c, m in marks.items()}
        check_poisoned(run_prefix(q, kp, vp2, ko, vo, plen.cuda(), olen.cuda(), True), want, sees, marks)


@pytest.mark.parametrize("D", [64, 72, 128, 200, 256])
def test_row_waves_infinite_values_in_slices(D):
    """And where four waves divide 128 rows and two workgroups or more a block's keys."""
    g = gen(18, D)
    B, T, N, Hq, Hk = 2, 512, 20000, 8, 1
    q, k, v = randn(g, (B, T, Hq, D), BF), randn(g, (B, N, Hk, D), BF), randn(g, (B, N, Hk, D), BF)
    assert rm.span_attention_workspace(q, k).numel() > 0
    span = torch.zeros((B, T, 2), dtype=torch.int32)
    span[..., 1] = torch.randint(0, N + 1, (B, T), generator=g, dtype=torch.int32)
    span[0, :, 0] = torch.randint(0, N, (T,), generator=g, dtype=torch.int32)
    j = torch.arange(N)
    seen = (j >= span[..., :1]) & (j < span[..., 1:])
    want = run_span(q, k, v, span.cuda())
    v2, marks = poisoned(v, [(0, i) for i in range(7, N, 4099)] + [(1, 9000), (1, 17777)])
    check_poisoned(run_span(q, k, v2, span.cuda()), want, seen, marks)


def check_one_column_each(run, v, key, sees):
    """v [B][N][Hk][D] with an infinity in one column of `key`, another one in every sample (8 b): rows that see the key
    (sees [T]) get it there, and nothing else changes."""
    B, D = v.shape[0], v.shape[-1]
    want = run(v)
    v2, at = v.clone(), torch.arange(B)
    v2[at, key, :, 8 * at % D] = float("inf")
    got = run(v2)
    expected = want.clone()
    for b in range(B):
        expected[b, sees, :, 8 * b % D] = float("inf")
    assert torch.equal(got, expected)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 72, 128, 200, 256])
@pytest.mark.parametrize("start,N", [(0, 128), (30, 128), (40, 300), (66, 128), (100, 128), (225, 300), (100, 9000)])
def test_one_wave_has_the_unseen_key(dtype, D, start, N):
    """Rows whose keys end inside the 32 of one wave, the other waves' being all seen or all unseen: an infinity there, in
    each column, which another wave may join."""
    g = gen(29, D, start, N)
    B, T, H = D // 8, 20, 2
    q, k, v = randn(g, (B, T, H, D), dtype), randn(g, (B, N, H, D), dtype), randn(g, (B, N, H, D), dtype)
    span = torch.empty((B, T, 2), dtype=torch.int32, device="cuda")
    rm.rm_attn_spans(span, N, q_start=torch.full((B,), start, dtype=torch.int32, device="cuda"))
    check_one_column_each(lambda x: run_span(q, k, x, span), v, start + T // 2, torch.arange(T) >= T // 2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 72, 128, 200, 256])
@pytest.mark.parametrize("P,S", [(128, 128), (0, 100), (300, 65), (4000, 128)])
def test_one_wave_has_the_unseen_own_key(dtype, D, P, S):
    g = gen(33, D, P, S)
    B, T, H = D // 8, 32, 1
    q, kp, vp, ko, vo = make_prefix(g, 1, B, T, P, S, H, H, D, dtype)
    q = q * 0.5
    check_one_column_each(lambda x: run_prefix(q, kp, vp, ko, x, None, None, True), vo, S - 10, torch.arange(T) >= T - 10)


@pytest.mark.parametrize("dtype,T,D", [(BF, 2048, 128), (BF, 850, 256), (F32, 1024, 64)])
def test_time_with_nan_values(dtype, T, D):
    """Values that are NaN throughout take a bounded number of passes: 5 to 12 times the usual time measured, a key at a
    time it was thousands."""
    g = gen(19, T, D)
    q, k, v = randn(g, (1, T, 8, D), dtype), randn(g, (1, T, 2, D), dtype), randn(g, (1, T, 2, D), dtype)
    span = torch.empty((1, T, 2), dtype=torch.int32, device="cuda")
    rm.rm_attn_spans(span, T)
    out, ws = torch.empty_like(q), rm.span_attention_workspace(q, k)

    def ms(values):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for i in range(6):
            if i == 1:
                begin.record()
            rm.rm_span_attention(q, k, values, out, ws, span=span)
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end)

    usual = ms(v)
    slow = ms(torch.full_like(v, float("nan")))
    assert bool(out.isnan().all())
    assert slow < 100 * usual


# ---------------------------------------------------------------------------------------------- spans

@pytest.mark.parametrize("B,T,N", [(1, 1, 1), (2, 7, 7), (3, 300, 300), (2, 5, 260), (2, 600, 5000)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("window", [0, 1, 50])
@pytest.mark.parametrize("docs", [0, 1, 30])
def test_spans(B, T, N, causal, window, docs):
    g = gen(30, T, N, causal, window, docs)
    doc = None
    if docs:
        doc = ((torch.rand((B, N), generator=g) < docs / N).int().cumsum(1, dtype=torch.int32) % 3 - int(docs > 1)).int().cuda()
    kv = torch.randint(-1, N + 2, (B,), generator=g, dtype=torch.int32).cuda()
    kv[0] = N
    start = torch.randint(-3, N, (B,), generator=g, dtype=torch.int32).cuda()
    start[0] = N - T
    pre = torch.randint(-1, N + 2, (B,), generator=g, dtype=torch.int32).cuda() if causal else None
    for args in ((None, None, None), (start, kv, pre)):
        span = torch.full((B, T, 2), -77, dtype=torch.int32, device="cuda")
        rm.rm_attn_spans(span, N, causal, window, *args, doc)
        ref = att.spans(B, T, N, causal, window, *(None if a is None else a.cpu().numpy() for a in args),
                        None if doc is None else doc.cpu().numpy())
        assert np.array_equal(span.cpu().numpy(), ref)


# ---------------------------------------------------------------------------------------------- norm and rotation

def rope_tol(ref, pos, freq, dtype, D, pairs):
    half = len(freq)
    r = np.abs(ref).copy()
    i, j = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if pairs else (np.arange(half), np.arange(half) + half)
    h = np.hypot(ref[..., i], ref[..., j])
    r[..., i], r[..., j] = h, h
    ang = np.zeros(ref.shape)
    a = 5 * 2.0 ** -53 * np.abs(pos.astype(np.float64)[:, None] * freq.astype(np.float64)[None, :])[:, None, :]
    ang[..., i], ang[..., j] = a, a
    return U[dtype] * np.abs(ref) + 1.5 * r * ((D / 2 + 24) * U32 + ang) + 1e-30


@pytest.mark.parametrize("src", [BF, F32])
@pytest.mark.parametrize("dst", [BF, F32])
@pytest.mark.parametrize("D,rot", [(8, 8), (64, 64), (64, 0), (72, 36), (80, 40), (128, 64), (200, 100), (256, 256), (256, 4)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("N", [1, 700])
def test_rope(src, dst, D, rot, pairs, N):
    g = gen(40, D, rot, pairs, N)
    Hq, Hk = 5, 2
    qkv = randn(g, (N, Hq + 2 * Hk, D), src)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    pos = torch.randint(0, 1 << 20, (N,), generator=g, dtype=torch.int32)
    pos[0], pos[-1] = -(1 << 31), (1 << 31) - 1
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float()
    gq, gk = randn(g, (D,), F32), randn(g, (D,), F32)
    rows = N + 3
    slot = torch.randperm(rows, generator=g)[:N].to(torch.int32)
    if N > 1:
        slot[1], slot[2], slot[3] = -1, rows, (1 << 31) - 1  # dropped
    for gains in ((gq, gk), (None, None)):
        qo = torch.full((N, Hq, D), float("nan"), dtype=dst, device="cuda")
        ko, vo = torch.full((rows, Hk, D), 3.0, dtype=dst, device="cuda"), torch.full((rows, Hk, D), 3.0, dtype=dst, device="cuda")
        rm.rm_qk_norm_rope(q, k, v, qo, ko, vo, pos.cuda(), freq.cuda() if rot else None, gains[0], gains[1], slot.cuda(),
                           1e-5, pairs)
        torch.cuda.synchronize()
        f = freq.numpy()[:rot // 2]
        p = pos.numpy()
        for x, gain, out, at in ((q, gains[0], qo, None), (k, gains[1], ko, slot.numpy())):
            ref = att.norm_rope(f64(x), None if gain is None else f64(gain), p, f, 1e-5, pairs)
            tol = rope_tol(ref, p, f, dst, D, pairs)
            if at is None:
                check(out, ref, tol)
                continue
            ok = (at >= 0) & (at < rows)
            full, ftol = np.full((rows, Hk, D), 3.0), np.zeros((rows, Hk, D))
            full[at[ok]], ftol[at[ok]] = ref[ok], tol[ok]
            check(out, full, ftol)
            vref = torch.full((rows, Hk, D), 3.0, dtype=dst, device="cuda")
            vref[torch.from_numpy(at[ok]).long().cuda()] = v[torch.from_numpy(ok).cuda()].to(dst)
            assert torch.equal(vo, vref)


@pytest.mark.parametrize("dst", [BF, F32])
def test_rope_without_values_slots_and_norm_of_zeros(dst):
    g = gen(41)
    q, k = randn(g, (33, 3, 64), F32), randn(g, (33, 1, 64), F32)
    q[4], k[5] = 0.0, 0.0
    one = torch.ones(64, device="cuda")
    qo, ko = torch.empty((33, 3, 64), dtype=dst, device="cuda"), torch.full((40, 1, 64), 9.0, dtype=dst, device="cuda")
    freq = torch.linspace(1, 0.001, 32, device="cuda")
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    rm.rm_qk_norm_rope(q, k, None, qo, ko, None, pos, freq, one, one)
    ref = att.norm_rope(f64(k), np.ones(64), np.arange(33), freq.cpu().numpy(), 1e-6, False)
    check(ko[:33], ref, rope_tol(ref, np.arange(33), freq.cpu().numpy(), dst, 64, False))
    assert not qo[4].any() and not ko[5].any() and bool((ko[33:] == 9.0).all())
    empty = torch.empty((0, 3, 64), dtype=F32, device="cuda")
    rm.rm_qk_norm_rope(empty, empty[:, :1], None, empty.to(dst), ko, None, pos[:0], freq)
    assert bool((ko[33:] == 9.0).all())


@pytest.mark.parametrize("dst", [BF, F32])
@pytest.mark.parametrize("N", [1, 5, 700])
@pytest.mark.parametrize("D", [64, 72])
def test_rope_into_one_buffer(dst, N, D):
    """Keys beside values in a cache's rows, heads and head-major planes, and all three in packed rows: the same bits as
    in tensors of their own, and nothing else written."""
    g = gen(42, N, D)
    Hq, Hk, rows = 6, 2, N + 3
    qkv = randn(g, (N, Hq + 2 * Hk, D), BF)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    pos = torch.randint(0, 5000, (N,), generator=g, dtype=torch.int32).cuda()
    slot = torch.randperm(rows, generator=g)[:N].to(torch.int32).cuda()
    freq, gain = torch.linspace(1, 0.001, D // 2, device="cuda"), randn(g, (D,), F32)

    def run(qo, ko, vo, at):
        for t in (qo, ko, vo):
            t.fill_(3.0)
        rm.rm_qk_norm_rope(q, k, v, qo, ko, vo, pos, freq, gain, gain, at)

    def new(*shape):
        return torch.full(shape, 7.0, dtype=dst, device="cuda")

    want = [new(N, Hq, D), new(rows, Hk, D), new(rows, Hk, D)]
    run(*want, slot)
    by_row, by_head, planes = new(rows, 2, Hk, D), new(rows, Hk, 2, D), new(Hk, 2, rows, D)
    for got in ([new(N, Hq, D), by_row[:, 0], by_row[:, 1]], [new(N, Hq, D), by_head[:, :, 0], by_head[:, :, 1]],
                [new(N, Hq, D), planes[:, 0].transpose(0, 1), planes[:, 1].transpose(0, 1)]):
        run(*got, slot)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    own = [new(N, Hq, D), new(N, Hk, D), new(N, Hk, D)]
    run(*own, None)
    packed = new(N, Hq + 2 * Hk + 1, D)
    run(packed[:, :Hq], packed[:, Hq:Hq + Hk], packed[:, Hq + Hk:-1], None)
    assert torch.equal(packed[:, :-1], torch.cat(own, 1)) and bool((packed[:, -1] == 7.0).all())


# ---------------------------------------------------------------------------------------------- together

def test_layer_of_an_observation_and_its_samples_in_a_graph():
    """An observation's rows through norm, rotation, spans and attention into a cache, then the action samples of a
    denoising step on that cache and their sparse FFN layer; captured, replayed with eager work in between, and every
    replay equal to the eager results; and on a stream of its own."""
    import workloads as wl
    from gpu_helpers import dev_weights

    g = gen(50)
    P, n, T, Hq, Hk, D, d, d_ff, cnt = 90, 3, 17, 8, 1, 64, 512, 1024, 300
    cache_k = torch.zeros((1, P, Hk, D), dtype=BF, device="cuda")
    cache_v = torch.zeros_like(cache_k)
    own_k = torch.zeros((n, T, Hk, D), dtype=BF, device="cuda")
    own_v = torch.zeros_like(own_k)
    obs, act = randn(g, (P, Hq + 2 * Hk, D), F32), randn(g, (n * T, Hq + 2 * Hk, D), F32)
    freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    gain = randn(g, (D,), F32, 0.1) + 1
    qo, qa = torch.empty((1, P, Hq, D), dtype=BF, device="cuda"), torch.empty((n, T, Hq, D), dtype=BF, device="cuda")
    oo, oa = torch.empty_like(qo), torch.empty_like(qa)
    pos = torch.arange(P + T, dtype=torch.int32, device="cuda")
    apos = pos[P:].repeat(n)
    span = torch.empty((1, P, 2), dtype=torch.int32, device="cuda")
    plen, olen = ints([70]), ints([T, T, T - 2])
    layer = dev_weights(wl.make_layer(50, 0, d, d_ff, "bf16", norm="random"))
    idx = torch.arange(d_ff, dtype=torch.int32, device="cuda").repeat(n)
    counts = ints([cnt] * n)
    x, y = torch.zeros((n, T, d), device="cuda"), torch.zeros((n, T, d), device="cuda")
    ws1 = rm.span_attention_workspace(qo, cache_k)
    ws2 = rm.prefix_attention_workspace(qa, cache_k, own_k)
    ws3 = rm.workspace(d, d_ff, rm.RM_BF16, n, T, cnt)

    def split(t):
        return t[:, :Hq], t[:, Hq:Hq + Hk], t[:, Hq + Hk:]

    def step():
        rm.rm_qk_norm_rope(*split(obs), qo[0], cache_k[0], cache_v[0], pos[:P], freq, gain, gain)
        rm.rm_attn_spans(span, P, causal=True, prefix_len=plen)
        rm.rm_span_attention(qo, cache_k, cache_v, oo, ws1, span=span)
        rm.rm_qk_norm_rope(*split(act), qa.view(n * T, Hq, D), own_k.view(n * T, Hk, D), own_v.view(n * T, Hk, D), apos,
                           freq, gain, gain)
        rm.rm_prefix_attention(qa, cache_k, cache_v, own_k, own_v, oa, ws2, own_len=olen)
        x.copy_(oa.view(n, T, Hq * D))
        rm.rm_sparse_ffn_layer(x, y, layer, idx, counts, cnt, ws3)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (qo, cache_k, cache_v, span, oo, qa, own_k, own_v, oa, y)]

    step()
    want = results()
    check_span(qo, cache_k, cache_v, span, out=oo)
    check_prefix((qa, cache_k, cache_v, own_k, own_v), None, olen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(3):
        for t in (qo, cache_k, own_k, oo, oa, y):
            t.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), want)), f"replay {r}"
        obs_q = randn(gen(51, r), (1, 4, 4, 64), BF)
        run_span(obs_q, obs_q, obs_q)
        torch.cuda.synchronize()


def test_two_streams_at_once():
    g = gen(52)
    sets = []
    for i in range(2):
        q, k, v = randn(g, (1, 1, 8, 128), BF), randn(g, (1, 20000, 2, 128), BF), randn(g, (1, 20000, 2, 128), BF)
        sets.append((q, k, v, run_span(q, k, v), torch.empty_like(q), rm.span_attention_workspace(q, k), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for q, k, v, _, out, ws, st in sets:
            rm.rm_span_attention(q, k, v, out, ws, stream=st)
    torch.cuda.synchronize()
    for s in sets:
        assert torch.equal(s[3], s[4])


def test_binding_refuses_wrong_tensors():
    x = torch.zeros((1, 4, 2, 64), dtype=BF, device="cuda")
    o = torch.zeros_like(x)
    with pytest.raises(ValueError):
        rm.rm_span_attention(x, x.float(), x, o, None)
    with pytest.raises(ValueError):
        rm.rm_span_attention(x.half(), x.half(), x.half(), o.half(), None)
    with pytest.raises(ValueError):
        rm.rm_span_attention(x, x[..., ::2], x[..., ::2], o, None)
    with pytest.raises(ValueError):
        rm.rm_span_attention(x, x, x, o, None, span=torch.zeros((1, 3, 2), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        rm.rm_prefix_attention(x.expand(3, 4, 2, 64), x.expand(2, 4, 2, 64), x.expand(2, 4, 2, 64), x.expand(3, 4, 2, 64),
                               x.expand(3, 4, 2, 64), torch.zeros((3, 4, 2, 64), dtype=BF, device="cuda"), None)
    with pytest.raises(rm.RmError) as e:
        rm.rm_span_attention(x, x, x, x, None)  # in place
    assert e.value.status == rm.RM_ERR_INVALID_ARG
    assert math.isfinite(float(x.float().sum()))
