"""The attention-side operators' measured calls: their inputs, plain forms, work and 64-bit results.

Four operators, the ones between two FFN layers of the action expert and of its VLM:

  qk_norm_rope      per-head RMSNorm and position rotation of queries and keys, keys and values into a cache
  attn_spans        masks (causal, prefix, window, documents, lengths) as one key interval per query row
  span_attention    attention over each row's interval, with capped scores or a distance bias
  prefix_attention  attention of a batch whose samples share a long prefix, plus each sample's own keys

run() computes the plain form in elementary torch operations in 32 bits (angles in 64), or with own = True makes the
library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
THETA = 10000.0


# ----------------------------------------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------------------------------------

def listed():
    return [
        # One sample's 51 action tokens of the action expert (8 query heads and 1 key head of 256), float32 projections
        # into bf16 queries and cache rows: the smallest call, once a layer and denoising step.
        dict(name="rope-action-51", op="rope", N=51, Hq=8, Hk=1, D=256, rot=256, src="f32", dst="bf16", norm=False,
             pairs=False, far=1024),
        # A VLM prefill of 850 rows (768 visual, 82 instruction and state rows).
        dict(name="rope-prefill-850", op="rope", N=850, Hq=8, Hk=1, D=256, rot=256, src="bf16", dst="bf16", norm=True,
             pairs=False, far=1024),
        # A long packed batch with grouped heads, half of each head rotated in adjacent pairs, far positions.
        dict(name="rope-packed-32k", op="rope", N=32768, Hq=32, Hk=8, D=128, rot=64, src="bf16", dst="bf16", norm=True,
             pairs=True, far=1000000),
        # The masks of one VLM prefill: a bidirectional prefix, causal rows behind it.
        dict(name="spans-prefill-850", op="spans", B=1, T=850, N=850, causal=True, prefix=True, window=0, docs=0, ragged=False),
        # The masks of a long packed batch of documents, padded at the end.
        dict(name="spans-docs-8x16k", op="spans", B=8, T=16384, N=16384, causal=True, prefix=False, window=0, docs=24, ragged=True),
        # The VLM's prefill attention at the framework's 850 rows.
        dict(name="span-prefill-850", op="span", B=1, T=850, N=850, Hq=8, Hk=1, D=256, dtype="bf16", cap=0.0, bias=False,
             mask="prefix"),
        # A long packed batch of documents, scores capped.
        dict(name="span-docs-16k", op="span", B=1, T=16384, N=16384, Hq=16, Hk=4, D=128, dtype="bf16", cap=50.0, bias=False,
             mask="docs"),
        # Single tokens of four sequences on long caches of ragged lengths, distance bias.
        dict(name="span-decode-128k", op="span", B=4, T=1, N=131072, Hq=32, Hk=4, D=128, dtype="bf16", cap=0.0, bias=True,
             mask="lens"),
        # float32, an odd length, a head width of no power of two (the vision tower's), window and bias.
        dict(name="span-f32-517", op="span", B=2, T=517, N=517, Hq=6, Hk=3, D=72, dtype="f32", cap=0.0, bias=True,
             mask="window"),
        # One action chunk on its observation's 850 rows: the smallest attention call of a denoising step.
        dict(name="prefix-action-1", op="prefix", groups=1, per=1, T=51, P=850, S=51, Hq=8, Hk=1, D=256, dtype="bf16",
             cap=0.0, causal=False, ragged=False),
        # 16 action samples of one observation.
        dict(name="prefix-action-16", op="prefix", groups=1, per=16, T=51, P=850, S=51, Hq=8, Hk=1, D=256, dtype="bf16",
             cap=0.0, causal=False, ragged=False),
        # Single tokens of 2 x 64 sequences behind two long shared prompts, each with its own ragged cache.
        dict(name="prefix-decode-128", op="prefix", groups=2, per=64, T=1, P=16384, S=512, Hq=32, Hk=8, D=128,
             dtype="bf16", cap=0.0, causal=True, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((8, 1), (16, 4), (32, 8), (6, 3), (4, 4), (12, 2))


def draw(rng):
    op = rng.choice(("rope", "spans", "span", "span", "prefix", "prefix"))
    Hq, Hk = rng.choice(HEADS)
    D = rng.choice((64, 72, 80, 128, 128, 256))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "rope":
        N = _log(rng, 1, 32768 * 40 * 128 // ((Hq + 2 * Hk) * D * 2))
        return dict(op=op, N=N, Hq=Hq, Hk=Hk, D=D, rot=rng.choice((D, D, D // 2 // 2 * 2)), src=rng.choice(("f32", "bf16")),
                    dst=dtype, norm=rng.random() < 0.5, pairs=rng.random() < 0.5, far=_log(rng, 64, 1000000))
    if op == "spans":
        B = rng.randint(1, 8)
        N = _log(rng, 1, 16384)
        docs = rng.choice((0, 1 + _log(rng, 1, 32)))
        return dict(op=op, B=B, T=N, N=N, causal=rng.random() < 0.8, prefix=docs == 0 and rng.random() < 0.5,
                    window=rng.choice((0, 0, _log(rng, 1, N))), docs=docs, ragged=rng.random() < 0.5)
    kind = rng.choice(("long", "few"))
    if op == "span":
        B = rng.randint(1, 4)
        if kind == "long":
            T = N = _log(rng, 1, 4096 if dtype == "bf16" else 1500)
            mask = rng.choice(("prefix", "docs", "window", "full"))
        else:
            T, N = rng.choice((1, 1, rng.randint(2, 9))), _log(rng, 16, 65536)
            mask = "lens"
        return dict(op=op, B=B, T=T, N=N, Hq=Hq, Hk=Hk, D=D, dtype=dtype, cap=rng.choice((0.0, 0.0, 30.0)),
                    bias=rng.random() < 0.4, mask=mask)
    causal = rng.random() < 0.5
    T = 1 if kind == "few" else _log(rng, 2, 96)
    return dict(op=op, groups=rng.randint(1, 3), per=_log(rng, 1, 24), T=T, P=_log(rng, 1, 4096 if kind == "long" else 12000),
                S=T + _log(rng, 1, 300), Hq=Hq, Hk=Hk, D=D, dtype=dtype, cap=rng.choice((0.0, 0.0, 30.0)), causal=causal,
                ragged=rng.random() < 0.5)


# ----------------------------------------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(DTYPES[dtype])


def _randint(g, lo, hi, shape):
    """Whole numbers in [lo, hi]."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _doc_ids(g, B, N, docs):
    """Ids of about `docs` documents of random lengths, in a row."""
    cuts = torch.rand((B, N), generator=g, device="cuda") < docs / N
    return cuts.to(torch.int32).cumsum(1, dtype=torch.int32)


def _mask_case(case):
    """The arguments of the masks that a span case's rows have, as a spans case."""
    m = case["mask"]
    return dict(B=case["B"], T=case["T"], N=case["N"], causal=m != "full", prefix=m == "prefix",
                window=max(1, case["N"] // 3) if m == "window" else 0, docs=6 if m == "docs" else 0, ragged=m == "lens")


def _mask_inputs(c, g):
    B, T, N = c["B"], c["T"], c["N"]
    s = dict(q_start=None, kv_len=None, prefix_len=None, doc=None)
    if c["ragged"]:
        s["kv_len"] = _randint(g, max(min(T, N), N - N // 4), N, (B,))
    if T != N:
        s["q_start"] = (s["kv_len"] - T).to(torch.int32) if c["ragged"] else torch.full((B,), N - T, dtype=torch.int32, device="cuda")
    if c["prefix"]:
        s["prefix_len"] = _randint(g, N // 2, N, (B,))
    if c["docs"]:
        s["doc"] = _doc_ids(g, B, N, c["docs"])
    return s


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "rope":
        N, Hq, Hk, D, rot = case["N"], case["Hq"], case["Hk"], case["D"], case["rot"]
        rows = N + 7
        # Queries, keys and values lie side by side in the rows of one projection's output.
        qkv = _randn(g, (N, Hq + 2 * Hk, D), case["src"])
        s = dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hk], v=qkv[:, Hq + Hk:],
                 pos=_randint(g, 0, case["far"] - 1, (N,)),
                 inv_freq=(THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)).float(),
                 slot=torch.randperm(rows, generator=g, device="cuda")[:N].to(torch.int32),
                 q_out=torch.empty((N, Hq, D), dtype=DTYPES[case["dst"]], device="cuda"),
                 k_out=_randn(g, (rows, Hk, D), case["dst"]), v_out=_randn(g, (rows, Hk, D), case["dst"]),
                 gain_q=None, gain_k=None)
        if case["norm"]:
            s["gain_q"] = 1.0 + 0.1 * _randn(g, (D,), "f32")
            s["gain_k"] = 1.0 + 0.1 * _randn(g, (D,), "f32")
    elif op == "spans":
        s = _mask_inputs(case, g)
        s["span"] = torch.empty((case["B"], case["T"], 2), dtype=torch.int32, device="cuda")
    elif op == "span":
        B, T, N, Hq, Hk, D, dt = (case[k] for k in ("B", "T", "N", "Hq", "Hk", "D", "dtype"))
        m = _mask_case(case)
        s = _mask_inputs(m, g)
        s.update(q=_randn(g, (B, T, Hq, D), dt, 2.0), k=_randn(g, (B, N, Hk, D), dt), v=_randn(g, (B, N, Hk, D), dt),
                 out=torch.empty((B, T, Hq, D), dtype=DTYPES[dt], device="cuda"), slopes=None, scale=D ** -0.5)
        if case["bias"]:  # a geometric row of slopes, one a head
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda", dtype=torch.float32) / Hq)
        # The masks as the attention takes them: made once for a batch, read by each of its layers.
        s["span"] = _plain_spans(m, s)
    else:
        G, n, T, P, S, Hq, Hk, D, dt = (case[k] for k in ("groups", "per", "T", "P", "S", "Hq", "Hk", "D", "dtype"))
        B = G * n
        s = dict(q=_randn(g, (B, T, Hq, D), dt, 2.0),
                 k_prefix=_randn(g, (G, P, Hk, D), dt), v_prefix=_randn(g, (G, P, Hk, D), dt),
                 k_own=_randn(g, (B, S, Hk, D), dt), v_own=_randn(g, (B, S, Hk, D), dt),
                 out=torch.empty((B, T, Hq, D), dtype=DTYPES[dt], device="cuda"), prefix_len=None, own_len=None,
                 scale=D ** -0.5)
        if case["ragged"]:
            s["prefix_len"] = _randint(g, P - P // 4, P, (G,))
            s["own_len"] = _randint(g, min(T, S), S, (B,))
    s["case"] = case
    return s


# ----------------------------------------------------------------------------------------------------------
# Plain forms
# ----------------------------------------------------------------------------------------------------------

def _norm_rotate(x, gain, cos, sin, rot, pairs):
    x = x.float()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
    r = x[..., :rot]
    if pairs:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((r, x[..., rot:]), -1)


def _plain_rope(s):
    c = s["case"]
    ang = (s["pos"].double()[:, None] * s["inv_freq"].double())[:, None, :]
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    slot = s["slot"].long()
    s["q_out"].copy_(_norm_rotate(s["q"], s["gain_q"], cos, sin, c["rot"], c["pairs"]))
    s["k_out"].index_copy_(0, slot, _norm_rotate(s["k"], s["gain_k"], cos, sin, c["rot"], c["pairs"]).to(s["k_out"].dtype))
    s["v_out"].index_copy_(0, slot, s["v"].to(s["v_out"].dtype))
    return s["q_out"], s["k_out"], s["v_out"]


def _plain_spans(c, s):
    B, T, N = c["B"], c["T"], c["N"]
    dev = "cuda"
    start = s["q_start"] if s["q_start"] is not None else torch.zeros((B,), dtype=torch.int32, device=dev)
    kv = s["kv_len"] if s["kv_len"] is not None else torch.full((B,), N, dtype=torch.int32, device=dev)
    p = start[:, None] + torch.arange(T, dtype=torch.int32, device=dev)
    lo = torch.zeros_like(p)
    hi = kv[:, None].expand(B, T)
    if c["causal"]:
        end = p + 1
        if s["prefix_len"] is not None:
            end = torch.maximum(end, s["prefix_len"][:, None])
        hi = torch.minimum(hi, end)
    if c["window"]:
        lo = torch.clamp(p - c["window"] + 1, min=0)
    inside = (p >= 0) & (p < kv[:, None])
    if s["doc"] is not None:
        doc = s["doc"]
        at = torch.arange(N, dtype=torch.int32, device=dev).expand(B, N)
        new = torch.ones_like(doc, dtype=torch.bool)
        new[:, 1:] = doc[:, 1:] != doc[:, :-1]
        last = torch.ones_like(new)
        last[:, :-1] = new[:, 1:]
        begin = torch.where(new, at, torch.zeros_like(at)).cummax(1).values
        ends = torch.where(last, at + 1, torch.full_like(at, N)).flip(1).cummin(1).values.flip(1)
        at_p = p.clamp(0, N - 1).long()
        lo = torch.maximum(lo, begin.gather(1, at_p))
        hi = torch.minimum(hi, ends.gather(1, at_p))
        inside = inside & (doc.gather(1, at_p) >= 0)
    empty = hi <= lo
    if c["causal"] or s["doc"] is not None:
        empty = empty | ~inside
    zero = torch.zeros_like(p)
    return torch.stack((torch.where(empty, zero, lo), torch.where(empty, zero, hi)), -1).to(torch.int32)


def _softmax_values(scores, seen, v):
    """softmax of the seen scores times v; rows that see nothing give 0."""
    scores = scores.masked_fill(~seen, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p / torch.where(total == 0, torch.ones_like(total), total), v)


def _capped(scores, cap):
    return cap * torch.tanh(scores / cap) if cap else scores


def _plain_span(s):
    c = s["case"]
    B, T, N, Hq, Hk, D = (c[k] for k in ("B", "T", "N", "Hq", "Hk", "D"))
    G = Hq // Hk
    q = s["q"].float().view(B, T, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * T, D)
    k = s["k"].float().permute(0, 2, 1, 3)
    v = s["v"].float().permute(0, 2, 1, 3)
    scores = _capped(torch.matmul(q, k.transpose(2, 3)) * s["scale"], c["cap"]).view(B, Hk, G, T, N)
    j = torch.arange(N, device="cuda")
    if s["slopes"] is not None:
        i = torch.arange(T, device="cuda")
        start = s["q_start"] if s["q_start"] is not None else torch.zeros((B,), dtype=torch.int32, device="cuda")
        dist = (start.long()[:, None, None] + i[:, None] - j).abs().float()
        scores = scores - s["slopes"].view(1, Hk, G, 1, 1) * dist[:, None, None]
    seen = (j >= s["span"][..., 0:1]) & (j < s["span"][..., 1:2])
    o = _softmax_values(scores, seen[:, None, None], v[:, :, None])
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D))
    return s["out"]


def _plain_prefix(s):
    c = s["case"]
    G, n, T, P, S, Hq, Hk, D = (c[k] for k in ("groups", "per", "T", "P", "S", "Hq", "Hk", "D"))
    B, R = G * n, Hq // Hk
    dev = "cuda"
    q = s["q"].float().view(G, n, T, Hk, R, D).permute(0, 3, 1, 4, 2, 5)  # [G][Hk][n][R][T][D]
    kp, vp = s["k_prefix"].float().permute(0, 2, 3, 1), s["v_prefix"].float().permute(0, 2, 1, 3)
    ko = s["k_own"].float().view(G, n, S, Hk, D).permute(0, 3, 1, 4, 2)  # [G][Hk][n][D][S]
    vo = s["v_own"].float().view(G, n, S, Hk, D).permute(0, 3, 1, 2, 4)
    sp = torch.matmul(q.reshape(G, Hk, n * R * T, D), kp).view(G, Hk, n, R, T, P)
    so = torch.matmul(q.reshape(G, Hk, n, R * T, D), ko).view(G, Hk, n, R, T, S)
    scores = _capped(torch.cat((sp, so), -1) * s["scale"], c["cap"])
    plen = s["prefix_len"] if s["prefix_len"] is not None else torch.full((G,), P, dtype=torch.int32, device=dev)
    olen = s["own_len"] if s["own_len"] is not None else torch.full((B,), S, dtype=torch.int32, device=dev)
    seen_p = (torch.arange(P, device=dev) < plen[:, None]).view(G, 1, 1, 1, 1, P).expand(G, 1, n, 1, T, P)
    j = torch.arange(S, device=dev)
    end = olen[:, None].expand(B, T)
    if c["causal"]:
        end = torch.minimum(end, olen[:, None] - T + torch.arange(T, device=dev) + 1)
    seen_o = (j < end[..., None]).view(G, 1, n, 1, T, S)
    scores = scores.masked_fill(~torch.cat((seen_p, seen_o), -1), float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    op = torch.matmul(p[..., :P].reshape(G, Hk, n * R * T, P), vp).view(G, Hk, n, R, T, D)
    oo = torch.matmul(p[..., P:].reshape(G, Hk, n, R * T, S), vo).view(G, Hk, n, R, T, D)
    s["out"].copy_((op + oo).permute(0, 2, 4, 1, 3, 5).reshape(B, T, Hq, D))
    return s["out"]


# ----------------------------------------------------------------------------------------------------------
# The library's calls
# ----------------------------------------------------------------------------------------------------------

def _own_run(s):
    import paper_2609_19104_amd as rm

    c = s["case"]
    op = c["op"]
    if op == "rope":
        rm.rm_qk_norm_rope(s["q"], s["k"], s["v"], s["q_out"], s["k_out"], s["v_out"], s["pos"], s["inv_freq"],
                           gain_q=s["gain_q"], gain_k=s["gain_k"], slot=s["slot"], eps=1e-6, pairs=c["pairs"])
        return s["q_out"], s["k_out"], s["v_out"]
    if op == "spans":
        rm.rm_attn_spans(s["span"], c["N"], causal=c["causal"], window=c["window"], q_start=s["q_start"],
                         kv_len=s["kv_len"], prefix_len=s["prefix_len"], doc=s["doc"])
        return s["span"]
    if op == "span":
        if "ws" not in s:
            s["ws"] = rm.span_attention_workspace(s["q"], s["k"])
        rm.rm_span_attention(s["q"], s["k"], s["v"], s["out"], s["ws"], span=s["span"], slopes=s["slopes"],
                             q_start=s["q_start"], scale=s["scale"], softcap=c["cap"])
        return s["out"]
    if "ws" not in s:
        s["ws"] = rm.prefix_attention_workspace(s["q"], s["k_prefix"], s["k_own"])
    rm.rm_prefix_attention(s["q"], s["k_prefix"], s["v_prefix"], s["k_own"], s["v_own"], s["out"], s["ws"],
                           prefix_len=s["prefix_len"], own_len=s["own_len"], causal=c["causal"], scale=s["scale"],
                           softcap=c["cap"])
    return s["out"]


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "rope":
        return _plain_rope(state)
    if op == "spans":
        return _plain_spans(state["case"], state)
    if op == "span":
        return _plain_span(state)
    return _plain_prefix(state)


# ----------------------------------------------------------------------------------------------------------
# Work
# ----------------------------------------------------------------------------------------------------------

def _span_pairs(c):
    """About how many (row, key) pairs the masks of a span case leave, of one sample."""
    T, N, m = c["T"], c["N"], c["mask"]
    if m == "full":
        return T * N
    if m == "lens":
        return T * N * 7 / 8
    if m == "prefix":  # prefix lengths spread evenly over [N / 2, N]: f N rows see f N keys, the rest see up to their own
        return N * N * (7 / 12 + (1 - 7 / 12) / 2)
    if m == "window":
        w = max(1, N // 3)
        return N * w - w * w / 2
    return N * N / 2 * 2 / 7 if N > 14 else N  # seven documents of random lengths


def work(case):
    op = case["op"]
    if op == "rope":
        n = case["N"] * (case["Hq"] + 2 * case["Hk"]) * case["D"]
        return {"bytes": n * (BYTES[case["src"]] + BYTES[case["dst"]]) + 8 * case["N"], "flops": 8 * n}
    if op == "spans":
        return {"bytes": case["B"] * case["T"] * 8 + (case["B"] * case["N"] * 4 if case["docs"] else 0), "flops": 0}
    e = BYTES[case["dtype"]]
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if op == "span":
        keys = case["N"] * (7 / 8 if case["mask"] == "lens" else 1)
        return {"bytes": case["B"] * (2 * case["T"] * Hq + 2 * keys * Hk) * D * e,
                "flops": 4 * D * Hq * case["B"] * _span_pairs(case)}
    B = case["groups"] * case["per"]
    P = case["P"] * (7 / 8 if case["ragged"] else 1)
    S = (case["S"] + min(case["T"], case["S"])) / 2 if case["ragged"] else case["S"]
    own_pairs = case["T"] * S - (case["T"] * (case["T"] - 1) / 2 if case["causal"] else 0)
    return {"bytes": (2 * B * case["T"] * Hq + 2 * (case["groups"] * P + B * S) * Hk) * D * e,
            "flops": 4 * D * Hq * B * (case["T"] * P + own_pairs)}


# ----------------------------------------------------------------------------------------------------------
# 64-bit results, from the definitions, one head or sample at a time
# ----------------------------------------------------------------------------------------------------------

def _exact_rope(c, s):
    half = c["rot"] // 2
    turn = torch.outer(s["pos"].double(), s["inv_freq"].double())
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + half)

    def heads(x, gain):
        y = x.double().clone()
        if gain is not None:
            y = y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * gain.double()
        z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(turn), turn)[:, None]
        y[..., first], y[..., second] = z.real.clone(), z.imag.clone()
        return y

    k, v = s["k_out"].double(), s["v_out"].double()
    k[s["slot"].long()] = heads(s["k"], s["gain_k"])
    v[s["slot"].long()] = s["v"].double()
    return heads(s["q"], s["gain_q"]), k, v


def _exact_row_block(q, k, v, seen, scale, cap, bias):
    x = q.double() @ k.double().T * scale
    if cap:
        x = torch.tanh(x / cap) * cap
    if bias is not None:
        x = x + bias
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, -1, keepdim=True)
    return torch.where(seen, torch.exp(x - lse), torch.zeros_like(x)) @ v.double()


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op == "rope":
        return _exact_rope(case, s)
    if op == "spans":
        return None
    Hq, Hk = case["Hq"], case["Hk"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if op == "span":
        j = torch.arange(case["N"], device="cuda")
        for b in range(case["B"]):
            seen = (j >= s["span"][b, :, :1]) & (j < s["span"][b, :, 1:])
            at = torch.arange(case["T"], device="cuda") + (int(s["q_start"][b]) if s["q_start"] is not None else 0)
            dist = (at[:, None] - j).abs().double()
            for h in range(Hq):
                bias = -s["slopes"][h].double() * dist if s["slopes"] is not None else None
                kv = h // (Hq // Hk)
                out[b, :, h] = _exact_row_block(s["q"][b, :, h], s["k"][b, :, kv], s["v"][b, :, kv], seen, s["scale"],
                                                case["cap"], bias)
        return out
    T, n = case["T"], case["per"]
    for b in range(case["groups"] * n):
        g = b // n
        P = int(s["prefix_len"][g]) if s["prefix_len"] is not None else case["P"]
        S = int(s["own_len"][b]) if s["own_len"] is not None else case["S"]
        k = torch.cat((s["k_prefix"][g, :P], s["k_own"][b, :S]))
        v = torch.cat((s["v_prefix"][g, :P], s["v_own"][b, :S]))
        j = torch.arange(P + S, device="cuda")
        end = P + S - T + torch.arange(T, device="cuda") + 1 if case["causal"] else torch.full((T,), P + S, device="cuda")
        seen = (j < P) | (j < end[:, None])
        for h in range(Hq):
            kv = h // (Hq // Hk)
            out[b, :, h] = _exact_row_block(s["q"][b, :, h], k[:, kv], v[:, kv], seen, s["scale"], case["cap"], None)
    return out
