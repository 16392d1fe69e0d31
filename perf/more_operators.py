"""Timed operators of attention whose scores are capped, biased by distance and masked by spans, in
training and in serving.

Every query sees one run of keys, its span: lo <= j < hi.  Spans say which document of a packed
sequence a token belongs to, which prefix all of a document's tokens see, and which rows are
padding.  A score is s = scale q.k, capped to c tanh(s / c), less slope_h |i - j|.  A case is one
operator ("op") at one size:

  fwd     O and LSE of every query over its span (``attn_span_fwd``)
  bwd     its backward: dQ, dK, dV from O, LSE and dO (``attn_span_bwd``)
  decode  the same scores for one new token per sequence over a paged cache, the sequences in
          groups that share a prefix, whose keys are read once for the group
          (``attn_decode_shared``)

Where ``own`` is false ``run`` computes them in elementary torch operations, in 32 bits, rounded
once at the end; where it is true it calls the library.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3 = torch.float8_e4m3fn
E_MIN = -110     # least exponent of a row's scale in the 8-bit cache


# ------------------------------------------------------------------ cases
def _attn(name, op, b, S, n_q, n_k, d, docs=0, prefix=0, pad=0, cap=0.0, bias=False, fused=False):
    """docs: mean length of a document (0: one), prefix: tokens at its start that all of it sees,
    pad: rows at the end of every sequence but the first that belong to none."""
    return {"name": name, "op": op, "b": b, "S": S, "n_q": n_q, "n_k": n_k, "d": d, "docs": docs,
            "prefix": prefix, "pad": pad, "cap": cap, "bias": bias, "fused": fused}


def _decode(name, b, groups, prefix, own_len, n_q, n_k, d, page, cache, cap=0.0, bias=False):
    return {"name": name, "op": "decode", "b": b, "groups": groups, "prefix": prefix,
            "own_len": own_len, "n_q": n_q, "n_k": n_k, "d": d, "page": page, "cache": cache,
            "cap": cap, "bias": bias}


def listed():
    return [
        # the least: a short sequence of one share's heads, every part of the score
        _attn("fwd_short_d64", "fwd", 1, 129, 4, 1, 64, prefix=17, cap=30.0, bias=True),
        # a ragged packed batch out of a fused projection's rows, prefixes and padding
        _attn("fwd_packed_d96", "fwd", 3, 1537, 7, 1, 96, docs=300, prefix=64, pad=200, cap=50.0,
              fused=True),
        # 16K tokens of packed documents, 8 heads on 2: what a packed training sequence looks like
        _attn("fwd_packed_s16k", "fwd", 1, 16384, 8, 2, 128, docs=2048, bias=True),
        # one document of 32K tokens, capped: the whole triangle
        _attn("fwd_cap_s32k", "fwd", 1, 32768, 4, 1, 128, cap=50.0),
        # the tiny share, every part of the score
        _attn("bwd_tiny", "bwd", 2, 512, 4, 4, 64, docs=150, prefix=20, pad=30, cap=30.0, bias=True),
        # a ragged batch with a prefix and padding
        _attn("bwd_prefix_d80", "bwd", 2, 2999, 7, 1, 80, docs=1200, prefix=256, pad=100, cap=50.0),
        # 16K tokens of packed documents
        _attn("bwd_packed_s16k", "bwd", 1, 16384, 8, 2, 128, docs=2048, bias=True),
        # one document of 16K tokens, capped: the largest
        _attn("bwd_cap_s16k", "bwd", 1, 16384, 8, 2, 128, cap=50.0),
        # a few short sequences, one dead slot, one too short for the prefix: latency
        _decode("decode_short_d80", 6, 2, 60, 40, 7, 1, 80, 16, "bf16", cap=30.0, bias=True),
        # 32 answers to one prompt of 16K tokens
        _decode("decode_b32_p16k", 32, 1, 16384, 500, 8, 2, 128, 64, "bf16"),
        # four system prompts in an 8-bit cache, 64 sequences
        _decode("decode_b64_g4_e4m3", 64, 4, 8000, 1000, 8, 2, 128, 64, "e4m3", bias=True),
        # 64 sequences on one context of 32K tokens, capped, 8 heads on 1
        _decode("decode_b64_p32k_cap", 64, 1, 32768, 1500, 8, 1, 128, 64, "bf16", cap=50.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    d = rng.choice([64, 80, 96, 128, 128])
    op = rng.choice(["fwd", "bwd", "decode"])
    cap, bias = rng.choice([0.0, 15.0, 30.0, 50.0]), rng.random() < 0.5
    if op != "decode":
        n_q, n_k = rng.choice([(8, 2), (8, 1), (7, 1), (4, 4), (2, 1), (4, 1), (16, 2)])
        b = rng.choice([1, 1, 2, 3, _log(rng, 1, 16)])
        pairs = (4 * 32768 ** 2 if op == "fwd" else 8 * 16384 ** 2) * 128 // d
        S = _log(rng, 1, min(32768, int((pairs / (b * n_q)) ** 0.5)))
        docs = rng.choice([0, _log(rng, 1, S), _log(rng, 1, S)])
        prefix = rng.choice([0, 0, _log(rng, 1, docs or S)])
        pad = rng.choice([0, S // 5]) if b > 1 else 0
        return _attn(None, op, b, S, n_q, n_k, d, docs, prefix, pad, cap, bias, rng.random() < 0.3)
    n_k, rep = rng.choice([1, 1, 2, 4]), rng.choice([1, 2, 4, 7, 8, 16])
    b = _log(rng, 1, 128)
    own_len = _log(rng, 1, 2000)
    prefix = _log(rng, 1, max(2, min(32768, 64 * 34000 // (b * n_k) - own_len)))
    return _decode(None, b, min(b, _log(rng, 1, 16)), prefix, own_len, n_k * rep, n_k, d,
                   rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"]), cap, bias)


# ------------------------------------- documents and lengths, fixed by the case
def _rng(c):
    return random.Random("-".join(str(c[k]) for k in sorted(c) if k != "name"))


def _documents(c):
    """Of every sequence the (first token, end) of its documents."""
    r, out = _rng(c), []
    for s in range(c["b"]):
        end = c["S"] - (c["pad"] if s else 0)
        at, docs = 0, []
        while at < end:
            n = end - at if c["docs"] == 0 else min(end - at, 1 + int(r.expovariate(1 / c["docs"])))
            docs.append((at, at + n))
            at += n
        out.append(docs)
    return out


def _groups(c):
    """(first sequence of every group and b, prefix length of every group, length of every
    sequence)."""
    r, b, n = _rng(c), c["b"], c["groups"]
    cuts = [0] + sorted(r.sample(range(1, b), n - 1)) + [b]
    prefix = [c["prefix"]] + [r.randint(0, c["prefix"]) for _ in range(n - 1)]
    lens = []
    for g in range(n):
        lens += [prefix[g] + r.randint(1, c["own_len"]) for _ in range(cuts[g + 1] - cuts[g])]
    if b >= 4:  # an empty slot, and a sequence that ends inside its group's prefix
        lens[1] = 0
        lens[2] = max(1, prefix[next(g for g in range(n) if cuts[g + 1] > 2)] // 2)
    return cuts, prefix, lens


# ----------------------------------------------------------------- inputs
def _spans(c):
    """int32 [b, S, 2]: lo and hi of every token."""
    rows = torch.zeros(c["b"], c["S"], 2, dtype=torch.int32)
    for s, docs in enumerate(_documents(c)):
        for lo, end in docs:
            rows[s, lo:end, 0] = lo
            hi = torch.arange(lo + 1, end + 1, dtype=torch.int32)
            rows[s, lo:end, 1] = hi.clamp(min=min(end, lo + c["prefix"]))
    return rows.cuda()


def _slopes(n):
    return 2.0 ** (-8.0 * torch.arange(1, n + 1, dtype=F32, device="cuda") / n)


def _pow2(e):
    """2^e in fp32, whole numbers -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(F32)


def _quantise(x):
    """A row (last axis) in e4m3 with a power-of-two scale: (values e4m3, scale bytes)."""
    x = x.float()
    m, ex = torch.frexp(x.abs().amax(-1))           # amax = m 2^ex, 0.5 <= m < 1
    e = (ex - 9 + (m > 0.875)).clamp(min=E_MIN)     # 448 = 0.875 * 2^9
    return (x * _pow2(-e)[..., None]).to(E4M3), (e + 127).to(torch.uint8)


def _cache(c, g):
    """Block table, pages and lengths of sequences whose groups hold their prefix's whole pages
    once; a page that the prefix ends in stands in every sequence's own copy."""
    cuts, prefix, lens = _groups(c)
    page, b = c["page"], c["b"]
    max_pages = -(-max(max(lens), max(prefix), 1) // page)
    table = torch.zeros(b, max_pages, dtype=torch.int64)
    n_pages, copies = 0, []
    for i, p in enumerate(prefix):
        whole = p // page
        shared = torch.arange(n_pages, n_pages + whole)
        n_pages += whole
        first = n_pages
        for s in range(cuts[i], cuts[i + 1]):
            table[s, :whole] = shared
            mine = max(0, max_pages - whole)
            table[s, whole:] = torch.arange(n_pages, n_pages + mine)
            if p % page and s > cuts[i]:
                copies.append((n_pages, first, p % page))
            n_pages += mine
    order = torch.randperm(max(1, n_pages), generator=g, device="cuda")
    out = {"table": order[table.cuda()].to(torch.int32)}
    shape = (max(1, n_pages), c["n_k"], page, c["d"])
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda", dtype=BF16)
        if copies:
            to, frm, n = (torch.tensor(v, device="cuda") for v in zip(*copies))
            old = torch.arange(page, device="cuda") < n[:, None]
            x[order[to]] = torch.where(old[:, None, :, None], x[order[frm]], x[order[to]])
        out[name + "_pages"], out[name + "_scales"] = (_quantise(x) if c["cache"] == "e4m3"
                                                       else (x, None))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out.update(lens=ints(lens), groups=ints(cuts), prefix_lens=ints(prefix),
               max_len=max_pages * page)
    return out


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=F32).to(BF16)  # noqa: E731
    b, n_q, n_k, d = c["b"], c["n_q"], c["n_k"], c["d"]
    st = {"case": c, "scale": d ** -0.5, "cap": c["cap"] or None,
          "slopes": _slopes(n_q) if c["bias"] else None}
    if c["op"] == "decode":
        st.update(_cache(c, g))
        st["q"] = randn(b, n_q, d) * 2
        return st
    S = c["S"]
    if c["fused"]:  # Q, K, V side by side, as one projection writes them
        qkv = randn(b, S, n_q + 2 * n_k, d)
        st["q"], st["k"] = qkv[:, :, :n_q], qkv[:, :, n_q:n_q + n_k]
        st["v"] = qkv[:, :, n_q + n_k:]
    else:
        st["q"], st["k"], st["v"] = randn(b, S, n_q, d) * 2, randn(b, S, n_k, d), randn(b, S, n_k, d)
    st["spans"] = _spans(c)
    if c["op"] == "bwd":  # what the forward left
        st["o"], st["lse"] = _forward(st)
        st["do"] = randn(b, S, n_q, d)
    return st


# ------------------------------------------------------------ plain forms
def _scores(st, s, dist):
    """Capped and biased scores of s = scale q.k ([b, n_k, rep, queries, keys]) in place, and the
    cap's derivative."""
    slope = None
    if st["cap"]:
        s.mul_(1 / st["cap"]).tanh_()
        slope = 1 - s * s
        s.mul_(st["cap"])
    if st["slopes"] is not None:
        n_k, rep = s.shape[1:3]
        s.sub_(st["slopes"].view(n_k, rep, 1, 1) * dist)
    return s, slope


def _heads_first(x, n_k):
    """[b, S, n, d] as fp32 [b, n_k, n/n_k * S, d]."""
    b, S, n, d = x.shape
    return x.float().permute(0, 2, 1, 3).reshape(b, n_k, n // n_k * S, d)


def _tokens_first(x, S):
    """[b, n_k, rep * S, d] as [b, S, n_k * rep, d]."""
    b, n_k, rows, d = x.shape
    return x.view(b, n_k * rows // S, S, d).transpose(1, 2)


def _square(st):
    """Scores of every query and key, the cap's derivative, and which are seen."""
    b, S, n_q, d = st["q"].shape
    n_k = st["k"].shape[2]
    at = torch.arange(S, device="cuda")
    s = _heads_first(st["q"], n_k) @ _heads_first(st["k"], n_k).transpose(2, 3)
    s = s.mul_(st["scale"]).view(b, n_k, n_q // n_k, S, S)
    s, slope = _scores(st, s, (at[:, None] - at).abs().float())
    lo, hi = st["spans"].long()[:, None, None, :, :, None].unbind(4)
    return s, slope, (at >= lo) & (at < hi)


def _forward(st):
    b, S, n_q, d = st["q"].shape
    n_k = st["k"].shape[2]
    s, _, seen = _square(st)
    s.masked_fill_(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    tot = p.sum(-1, keepdim=True)
    p.div_(torch.where(tot == 0, torch.ones_like(tot), tot))
    o = p.view(b, n_k, -1, S) @ _heads_first(st["v"], n_k)
    return _tokens_first(o, S).to(BF16).contiguous(), (m + tot.log()).view(b, n_q, S)


def _backward(st):
    b, S, n_q, d = st["q"].shape
    n_k = st["k"].shape[2]
    s, slope, seen = _square(st)
    lse = st["lse"].view(b, n_k, -1, S, 1)
    p = s.sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_()
    p.masked_fill_(~seen, 0.0)
    do = _heads_first(st["do"], n_k)
    dv = p.view(b, n_k, -1, S).transpose(2, 3) @ do
    dp = (do @ _heads_first(st["v"], n_k).transpose(2, 3)).view_as(p)
    dot = (do * _heads_first(st["o"], n_k)).sum(-1).view(b, n_k, -1, S, 1)
    ds = dp.sub_(dot).mul_(p).mul_(st["scale"])
    if slope is not None:
        ds.mul_(slope)
    ds = ds.view(b, n_k, -1, S)
    dq = ds @ _heads_first(st["k"], n_k)
    dk = ds.transpose(2, 3) @ _heads_first(st["q"], n_k)
    return tuple(_tokens_first(x, S).to(BF16).contiguous() for x in (dq, dk, dv))


def _gather(st, name):
    """Every sequence's tokens as its row of the table lists them, [b, n_k, L, d] in fp32."""
    pages = st[name + "_pages"]
    at = st["table"].long()
    x = (pages.view(torch.uint8)[at].view(E4M3) if pages.dtype == E4M3 else pages[at]).float()
    if pages.dtype == E4M3:
        x = x * _pow2(st[name + "_scales"][at].int() - 127)[..., None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _attend(st):
    q, lens = st["q"], st["lens"]
    b, n_q, d = q.shape
    K = _gather(st, "k")
    n_k, L = K.shape[1:3]
    at = torch.arange(L, device="cuda")
    s = (q.float().view(b, n_k, -1, d) @ K.transpose(2, 3)).mul_(st["scale"])[:, :, :, None]
    del K
    dist = (lens[:, None] - 1 - at).abs().float().view(b, 1, 1, 1, L)
    s, _ = _scores(st, s, dist)
    dead = (at >= lens[:, None])[:, None, None]
    s = s[:, :, :, 0].masked_fill_(dead, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    tot = p.sum(-1, keepdim=True)
    V = _gather(st, "v")
    o = (p @ V / tot).masked_fill_((lens == 0)[:, None, None, None], 0.0)
    return o.view(b, n_q, d).to(BF16), (m + tot.log()).view(b, n_q)


def run(state):
    st, op = state, state["case"]["op"]
    if own:
        return _run_own(st, op)
    return {"fwd": _forward, "bwd": _backward, "decode": _attend}[op](st)


def _run_own(st, op):
    import paper_2609_03151_amd as basp

    rule = {"scale": st["scale"], "cap": st["cap"], "slopes": st["slopes"]}
    if op == "fwd":
        return basp.attn_span_fwd(st["q"], st["k"], st["v"], st["spans"], **rule)
    if op == "bwd":
        return basp.attn_span_bwd(st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"],
                                  st["spans"], grad_dtype=BF16, **rule)
    return basp.attn_decode_shared(st["q"], st["k_pages"], st["v_pages"], st["table"], st["lens"],
                                   st["groups"], st["prefix_lens"], max_len=st["max_len"],
                                   k_scales=st["k_scales"], v_scales=st["v_scales"], **rule)


# ------------------------------------------------------------------- work
def work(case):
    c = case
    n_q, n_k, d = c["n_q"], c["n_k"], c["d"]
    if c["op"] != "decode":
        pairs = 0
        for docs in _documents(c):
            for lo, end in docs:
                n, p = end - lo, min(c["prefix"], end - lo)
                pairs += n * (n + 1) // 2 + p * (p - 1) // 2
        tokens = c["b"] * c["S"]
        rows = tokens * d * 2
        if c["op"] == "fwd":  # Q, K, V in, O and LSE out
            return {"bytes": rows * (2 * n_q + 2 * n_k) + tokens * (4 * n_q + 8),
                    "flops": 4 * pairs * n_q * d}
        return {"bytes": rows * (4 * n_q + 4 * n_k) + tokens * (4 * n_q + 8),
                "flops": 10 * pairs * n_q * d}
    cuts, prefix, lens = _groups(c)
    shared = own_keys = 0
    for g, p in enumerate(prefix):
        mine = lens[cuts[g]:cuts[g + 1]]
        shared += p if any(n >= p for n in mine) else 0
        own_keys += sum(n - p if n >= p else n for n in mine)
    row = d * (1 if c["cache"] == "e4m3" else 2) + (1 if c["cache"] == "e4m3" else 0)
    return {"bytes": 2 * n_k * (shared + own_keys) * row + c["b"] * n_q * (4 * d + 4)
            + 4 * (shared + own_keys) // c["page"],
            "flops": 4.0 * sum(lens) * n_q * d}


# ------------------------------------------------------------------ exact
def _rule(st, s, head, dist):
    """u and du/ds in fp64 of scores s of a query head at these distances."""
    one = torch.ones_like(s)
    if st["cap"]:
        e = torch.exp(-2 * s.abs() / st["cap"])
        u, one = torch.sign(s) * (1 - e) / (1 + e) * st["cap"], 4 * e / (1 + e) ** 2
    else:
        u = s
    if st["slopes"] is not None:
        u = u - st["slopes"][head].double() * dist
    return u, one


def _exact_rows(st, s, h, i0, i1):
    """Weights [rows, keys] of query head h, rows i0 .. i1 of sequence s, their LSE, the rule's
    derivative, and the keys they reach (a slice)."""
    rep = st["q"].shape[2] // st["k"].shape[2]
    lo, hi = st["spans"][s, i0:i1].long().unbind(1)
    live = hi > lo
    if not live.any():
        return None
    keys = slice(int(lo[live].min()), int(hi[live].max()))
    q = st["q"][s, i0:i1, h].double()
    k = st["k"][s, keys, h // rep].double()
    i = torch.arange(i0, i1, device="cuda")[:, None]
    j = torch.arange(keys.start, keys.stop, device="cuda")
    u, slope = _rule(st, torch.mm(q, k.t().contiguous()) * st["scale"], h, (i - j).abs().double())
    u = torch.where((j >= lo[:, None]) & (j < hi[:, None]), u, -math.inf)
    lse = torch.logsumexp(u, 1)
    return torch.where(live[:, None], torch.exp(u - lse[:, None]), 0.0), lse, slope, keys


def _exact_attn(c, st):
    b, S, n_q, d = st["q"].shape
    n_k = st["k"].shape[2]
    rep, scale = n_q // n_k, st["scale"]
    zeros = lambda n: torch.zeros(b, S, n, d, dtype=F64, device="cuda")  # noqa: E731
    o, dq, dk, dv = zeros(n_q), zeros(n_q), zeros(n_k), zeros(n_k)
    lse = torch.full((b, n_q, S), -math.inf, dtype=F64, device="cuda")
    for s in range(b):
        for h in range(n_q):
            for i0 in range(0, S, 4096):
                i1 = min(S, i0 + 4096)
                got = _exact_rows(st, s, h, i0, i1)
                if got is None:
                    continue
                p, lse[s, h, i0:i1], slope, keys = got
                v = st["v"][s, keys, h // rep].double()
                o[s, i0:i1, h] = torch.mm(p, v)
                if c["op"] == "fwd":
                    continue
                do = st["do"][s, i0:i1, h].double()
                dp = torch.mm(do, v.t().contiguous())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * slope * scale
                dq[s, i0:i1, h] = torch.mm(ds, st["k"][s, keys, h // rep].double())
                dk[s, keys, h // rep] += torch.mm(ds.t().contiguous(), st["q"][s, i0:i1, h].double())
                dv[s, keys, h // rep] += torch.mm(p.t().contiguous(), do)
    return (o, lse) if c["op"] == "fwd" else (dq, dk, dv)


def _exact_decode(c, st):
    b, n_q, d = st["q"].shape
    n_k, page = c["n_k"], c["page"]
    rep = n_q // n_k
    o = torch.zeros(b, n_q, d, dtype=F64, device="cuda")
    lse = torch.full((b, n_q), -math.inf, dtype=F64, device="cuda")
    for s, n in enumerate(_groups(c)[2]):
        if n == 0:
            continue
        at = st["table"][s, :-(-n // page)].long()
        dist = (n - 1 - torch.arange(n, device="cuda")).double()
        rows = []
        for name in ("k", "v"):
            x = st[name + "_pages"]
            x = x.view(torch.uint8)[at].view(E4M3).double() if x.dtype == E4M3 else x[at].double()
            if c["cache"] == "e4m3":
                e = st[name + "_scales"][at].long() - 127
                x = x * ((e + 1023) << 52).view(F64)[..., None]
            rows.append(x.transpose(0, 1).reshape(n_k, -1, d)[:, :n])
        for h in range(n_q):
            u, _ = _rule(st, torch.mv(rows[0][h // rep], st["q"][s, h].double()) * st["scale"], h,
                         dist)
            lse[s, h] = torch.logsumexp(u, 0)
            o[s, h] = torch.mv(rows[1][h // rep].t().contiguous(), torch.exp(u - lse[s, h]))
    return o, lse


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_decode(case, st) if case["op"] == "decode" else _exact_attn(case, st)
