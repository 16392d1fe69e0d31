"""Timed operators around a rank's attention: norm and rotation of queries and keys, the paged
key-value cache, and attention of one new token over it.

A case is one operator ("op") at one size:

  norm_rope      RMS norm of each query and key head with a learned weight, and the position
                 rotation, in one pass over Q and K (``qk_norm_rope``)
  norm_rope_bwd  its backward: gradients of Q, K and of both weights (``qk_norm_rope_bwd``)
  cache          K, V of T new tokens per sequence written into a paged cache, quantised where the
                 cache has 8 bits, and every sequence's tokens read back (``kv_write``, ``kv_read``)
  decode         attention of one new token per sequence over the paged cache (``attn_decode``)
  step           the three in a row, as one token is generated (norm and rotation, write, attention)

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
EPS = 1e-6
TYPES = {"bf16": BF16, "f32": F32, "e4m3": E4M3}
E_MIN = -110     # least exponent of a row's scale in the 8-bit cache


# ------------------------------------------------------------------ cases
def _norm(name, op, b, S, n_q, n_k, d, rot, dtype="bf16", grad="f32", interleaved=False,
          fused=False, pos0=0):
    return {"name": name, "op": op, "b": b, "S": S, "n_q": n_q, "n_k": n_k, "d": d, "rot": rot,
            "dtype": dtype, "grad": grad, "interleaved": interleaved, "fused": fused, "pos0": pos0}


def _cache(name, b, T, ctx, n_k, d, page, cache):
    return {"name": name, "op": "cache", "b": b, "T": T, "ctx": ctx, "n_k": n_k, "d": d,
            "page": page, "cache": cache}


def _decode(name, b, max_len, n_q, n_k, d, page, cache, lens="ragged", op="decode"):
    return {"name": name, "op": op, "b": b, "max_len": max_len, "n_q": n_q, "n_k": n_k, "d": d,
            "page": page, "cache": cache, "lens": lens}


def listed():
    return [
        # one new token of 16 sequences: a launch
        _norm("norm_rope_token", "norm_rope", 16, 1, 8, 2, 128, 128, pos0=4096),
        # a ragged batch out of a fused projection's rows, half the head rotated, paired (2i, 2i+1)
        _norm("norm_rope_fused_d96", "norm_rope", 3, 1037, 7, 1, 96, 48, interleaved=True,
              fused=True),
        # the Llama-3-70B share at 128K tokens
        _norm("norm_rope_s128k", "norm_rope", 1, 131072, 8, 1, 128, 128),
        # the tiny share in fp32 throughout
        _norm("norm_rope_bwd_tiny", "norm_rope_bwd", 2, 512, 4, 4, 64, 64, dtype="f32"),
        # the Llama-3-8B share at 32K tokens; fp32 gradients, as the attention backward gives them
        _norm("norm_rope_bwd_s32k", "norm_rope_bwd", 1, 32768, 8, 2, 128, 128),
        # five ragged prompts into small pages
        _cache("cache_ragged_d80", 5, 333, 1500, 1, 80, 16, "bf16"),
        # the last 8K tokens of a 32K prompt, quantised, and all of it read back
        _cache("cache_e4m3_s32k", 1, 8192, 24576, 2, 128, 64, "e4m3"),
        # short sequences, an empty one and one of a single token among them: latency
        _decode("decode_short_d80", 5, 77, 7, 1, 80, 16, "bf16"),
        # one long sequence: the Llama-3-70B share's heads over 128K tokens
        _decode("decode_one_s128k", 1, 131072, 8, 1, 128, 64, "bf16", lens="full"),
        # a serving batch of ragged sequences up to 32K tokens, in both cache types
        _decode("decode_b64_e4m3", 64, 32768, 8, 2, 128, 64, "e4m3"),
        _decode("decode_b64_bf16", 64, 32768, 8, 2, 128, 64, "bf16"),
        # a whole step for 32 sequences
        _decode("step_b32_s8k", 32, 8192, 8, 2, 128, 64, "bf16", op="step"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    d = rng.choice([64, 80, 96, 128, 128])
    op = rng.choice(["norm_rope", "norm_rope_bwd", "cache", "decode", "decode", "step"])
    if op.startswith("norm"):
        n_q, n_k = rng.choice([(8, 2), (8, 1), (7, 1), (4, 4), (2, 1), (32, 8), (28, 4)])
        rows = 131072 * 9 if op == "norm_rope" else 32768 * 10
        tokens = _log(rng, 1, rows * 128 // ((n_q + n_k) * d))
        b = min(tokens, _log(rng, 1, 64))
        return _norm(None, op, b, max(1, tokens // b), n_q, n_k, d, rng.choice([d, d, d // 2]),
                     rng.choice(["bf16", "bf16", "f32"]), rng.choice(["f32", "f32", "bf16"]),
                     rng.random() < 0.3, rng.random() < 0.3, rng.choice([0, 0, 1000]))
    n_k, rep = rng.choice([1, 1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8, 16])
    page, cache = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"])
    if op == "cache":
        b = _log(rng, 1, 32)
        T = _log(rng, 1, max(2, 65536 // (b * n_k)))
        ctx = rng.choice([0, _log(rng, 1, max(2, 65536 // (b * n_k) - T + 1))])
        return _cache(None, b, T, ctx, n_k, d, page, cache)
    b = _log(rng, 1, 128)
    most = 64 * 32768 * 2 if op == "decode" else 32 * 8192 * 2
    L = _log(rng, 1, min(131072, most // (b * n_k)))
    return _decode(None, b, L, n_k * rep, n_k, d, page, "bf16" if op == "step" else cache,
                   rng.choice(["ragged", "ragged", "full"]), op)


# -------------------------------------------------- lengths, fixed by the case
def _rng(c):
    return random.Random("-".join(str(c[k]) for k in sorted(c) if k != "name"))


def _lens(c):
    """Tokens of each sequence that a new token attends to (its own among them)."""
    b, L = c["b"], c["max_len"]
    if c["lens"] == "full":
        return [L] * b
    r = _rng(c)
    lens = [r.randint(1, L) for _ in range(b)]
    lens[0] = L
    if c["op"] == "decode" and b >= 4:
        lens[1], lens[2] = 0, 1
    return lens


def _starts(c):
    """(first position, number) of the new tokens of each sequence of a cache case."""
    r = _rng(c)
    if c["b"] == 1:
        return [c["ctx"]], [c["T"]]
    return ([r.randint(0, c["ctx"]) for _ in range(c["b"])],
            [c["T"]] + [r.randint(0, c["T"]) for _ in range(c["b"] - 1)])


# ----------------------------------------------------------------- inputs
def _table(n, rot, gen=None):
    """cos, sin [n, rot/2] in fp32, the angles formed in 64 bits."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device="cuda") / rot)
    ang = torch.arange(n, dtype=F64, device="cuda")[:, None] * freq
    return ang.cos().float(), ang.sin().float()


def _pow2(e):
    """2^e in fp32, whole numbers -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(F32)


def _quantise(x):
    """A row (last axis) in e4m3 with a power-of-two scale: (values e4m3, scale bytes)."""
    x = x.float()
    a = x.abs()
    amax = torch.where(a < math.inf, a, torch.zeros_like(a)).amax(-1)
    m, ex = torch.frexp(amax)                       # amax = m 2^ex, 0.5 <= m < 1
    e = ex - 9 + (m > 0.875)                        # 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(min=E_MIN)
    return (x * _pow2(-e)[..., None]).to(E4M3), (e + 127).to(torch.uint8)


def _pages(g, n_pages, n_k, page, d, cache):
    """K, V pages [n_pages, n_k, page, d] as a running program leaves them, and their scales."""
    out = []
    for _ in range(2):
        p = torch.randn(n_pages, n_k, page, d, generator=g, device="cuda", dtype=BF16)
        out.append(_quantise(p) if cache == "e4m3" else (p, None))
    return {"k_pages": out[0][0], "v_pages": out[1][0], "k_scales": out[0][1],
            "v_scales": out[1][1]}


def _block_table(g, b, max_pages):
    ids = torch.randperm(b * max_pages, generator=g, device="cuda")
    return ids.view(b, max_pages).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s, dtype=BF16: torch.randn(*s, generator=g, device="cuda", dtype=F32).to(dtype)  # noqa: E731
    weight = lambda: 1 + 0.1 * randn(c["d"], dtype=F32)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    d, b = c["d"], c["b"]
    st = {"case": c}
    if c["op"].startswith("norm"):
        S, n_q, n_k, dt = c["S"], c["n_q"], c["n_k"], TYPES[c["dtype"]]
        if c["fused"]:  # Q, K, V side by side, as one projection writes them
            qkv = randn(b, S, n_q + 2 * n_k, d, dtype=dt)
            st["q"], st["k"] = qkv[:, :, :n_q], qkv[:, :, n_q:n_q + n_k]
        else:
            st["q"], st["k"] = randn(b, S, n_q, d, dtype=dt), randn(b, S, n_k, d, dtype=dt)
        st["qw"], st["kw"] = weight(), weight()
        st["cos"], st["sin"] = _table(c["pos0"] + S, c["rot"])
        if c["op"] == "norm_rope_bwd":
            gt = TYPES[c["grad"]]
            st["dq"], st["dk"] = randn(b, S, n_q, d, dtype=gt), randn(b, S, n_k, d, dtype=gt)
        return st
    n_k, page = c["n_k"], c["page"]
    if c["op"] == "cache":
        T, L = c["T"], c["ctx"] + c["T"]
        mp = -(-L // page)
        st["table"] = _block_table(g, b, mp)
        st.update(_pages(g, b * mp, n_k, page, d, c["cache"]))
        st["k"], st["v"] = randn(b, T, n_k, d), randn(b, T, n_k, d)
        start, count = _starts(c)
        st["start"], st["count"] = ints(start), ints(count)
        st["total"] = ints([s + n for s, n in zip(start, count)])
        return st
    mp = -(-c["max_len"] // page)
    st["table"] = _block_table(g, b, mp)
    st.update(_pages(g, b * mp, n_k, page, d, c["cache"]))
    st["lens"] = ints(_lens(c))
    st["scale"] = d ** -0.5
    if c["op"] == "decode":
        st["q"] = randn(b, c["n_q"], d) * 1.5
    else:
        qkv = randn(b, 1, c["n_q"] + 2 * n_k, d)
        st["q"], st["k"] = qkv[:, :, :c["n_q"]], qkv[:, :, c["n_q"]:c["n_q"] + n_k]
        st["v"] = qkv[:, :, c["n_q"] + n_k:]
        st["qw"], st["kw"] = weight(), weight()
        st["cos"], st["sin"] = _table(c["max_len"], d)
        st["start"] = st["lens"] - 1
    return st


# ------------------------------------------------------------ plain forms
def _rotate(x, cos, sin, rot, interleaved):
    """x [b, S, n, d], cos and sin [b or 1, S, 1, rot/2], fp32."""
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., rot:]), -1) if rot < x.shape[-1] else y


def _angles(st, c, positions=None):
    if positions is None:
        sl = slice(c["pos0"], c["pos0"] + c["S"])
        return st["cos"][sl][None, :, None], st["sin"][sl][None, :, None]
    at = positions.long()
    return st["cos"][at][:, None, None], st["sin"][at][:, None, None]


def _norm_rope(x, w, cos, sin, rot, interleaved):
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    return _rotate(f * r * w, cos, sin, rot, interleaved).to(x.dtype)


def _norm_rope_bwd(x, dy, w, cos, sin, rot, interleaved):
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    z = _rotate(dy.float(), cos, -sin, rot, interleaved)
    g = z * w
    dx = r * (g - f * (r * r * (g * f).mean(-1, keepdim=True)))
    return dx.to(dy.dtype), (z * f * r).sum((0, 1, 2))


def _write(st, k, v, start, count):
    b, T, n_k, d = k.shape
    page = st["k_pages"].shape[2]
    at = start.long()[:, None] + torch.arange(T, device="cuda")
    if count is None:
        s, t = torch.meshgrid(torch.arange(b, device="cuda"), torch.arange(T, device="cuda"),
                              indexing="ij")
        s, t = s.reshape(-1), t.reshape(-1)
    else:
        s, t = torch.nonzero(torch.arange(T, device="cuda") < count[:, None], as_tuple=True)
    at = at[s, t]
    pid, off = st["table"].long()[s, at // page], at % page
    h = torch.arange(n_k, device="cuda")
    for x, name in ((k, "k"), (v, "v")):
        x = x[s, t]
        pages = st[name + "_pages"]
        if pages.dtype == E4M3:
            x, e = _quantise(x)
            st[name + "_scales"][pid[:, None], h, off[:, None]] = e
            pages, x = pages.view(torch.uint8), x.view(torch.uint8)
        pages[pid[:, None], h, off[:, None]] = x


def _gather(st, name, L):
    """The first L tokens of every sequence, [b, n_k, L, d] in fp32."""
    pages = st[name + "_pages"]
    at = st["table"].long()
    b = at.shape[0]
    x = (pages.view(torch.uint8)[at].view(E4M3) if pages.dtype == E4M3 else pages[at]).float()
    if pages.dtype == E4M3:
        x = x * _pow2(st[name + "_scales"][at].int() - 127)[..., None]
    _, n_k, page, d = pages.shape
    return x.permute(0, 2, 1, 3, 4).reshape(b, n_k, -1, d)[:, :, :L]


def _read(st, L, total):
    live = (torch.arange(L, device="cuda") < total[:, None])[:, :, None, None]
    out = [torch.where(live, _gather(st, n, L).permute(0, 2, 1, 3), 0.0).to(BF16)
           for n in ("k", "v")]
    return out


def _attend(q, st, L, scale):
    b, n_q, d = q.shape
    K = _gather(st, "k", L)
    n_k = K.shape[1]
    dead = (torch.arange(L, device="cuda") >= st["lens"][:, None])[:, None, None]
    s = (q.float().view(b, n_k, n_q // n_k, d) @ K.transpose(2, 3)) * scale
    del K
    s.masked_fill_(dead, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    del s
    tot = p.sum(-1, keepdim=True)
    V = _gather(st, "v", L).masked_fill_(dead.transpose(2, 3), 0.0)
    empty = (st["lens"] == 0)[:, None, None, None]
    o = (p @ V / tot).masked_fill_(empty, 0.0)
    return o.view(b, n_q, d).to(BF16), (m + tot.log()).view(b, n_q)


def run(state):
    st, c = state, state["case"]
    if own:
        return _run_own(st, c)
    if c["op"].startswith("norm"):
        args = (*_angles(st, c), c["rot"], c["interleaved"])
        if c["op"] == "norm_rope":
            return _norm_rope(st["q"], st["qw"], *args), _norm_rope(st["k"], st["kw"], *args)
        dq, dqw = _norm_rope_bwd(st["q"], st["dq"], st["qw"], *args)
        dk, dkw = _norm_rope_bwd(st["k"], st["dk"], st["kw"], *args)
        return dq, dk, dqw, dkw
    if c["op"] == "cache":
        _write(st, st["k"], st["v"], st["start"], st["count"])
        return tuple(_read(st, c["ctx"] + c["T"], st["total"]))
    if c["op"] == "decode":
        return _attend(st["q"], st, c["max_len"], st["scale"])
    args = (*_angles(st, c, st["start"]), c["d"], False)
    q = _norm_rope(st["q"], st["qw"], *args)
    k = _norm_rope(st["k"], st["kw"], *args)
    _write(st, k, st["v"], st["start"], None)
    o, lse = _attend(q[:, 0], st, c["max_len"], st["scale"])
    return o, lse, st["k_pages"], st["v_pages"]


def _run_own(st, c):
    import paper_2609_03151_amd as basp

    if c["op"].startswith("norm"):
        more = {"eps": EPS, "pos0": c["pos0"], "interleaved": c["interleaved"]}
        if c["op"] == "norm_rope":
            return basp.qk_norm_rope(st["q"], st["k"], st["qw"], st["kw"], st["cos"], st["sin"],
                                     **more)
        return basp.qk_norm_rope_bwd(st["q"], st["k"], st["dq"], st["dk"], st["qw"], st["kw"],
                                     st["cos"], st["sin"], **more)
    pages = (st["k_pages"], st["v_pages"], st["table"])
    scales = {"k_scales": st["k_scales"], "v_scales": st["v_scales"]}
    if c["op"] == "cache":
        basp.kv_write(st["k"], st["v"], *pages, st["start"], count=st["count"], **scales)
        return basp.kv_read(*pages, c["ctx"] + c["T"], count=st["total"], **scales)
    if c["op"] == "decode":
        return basp.attn_decode(st["q"], *pages, st["lens"], scale=st["scale"],
                                max_len=c["max_len"], **scales)
    q, k = basp.qk_norm_rope(st["q"], st["k"], st["qw"], st["kw"], st["cos"], st["sin"], eps=EPS,
                             positions=st["start"].view(-1, 1))
    basp.kv_write(k, st["v"], *pages, st["start"], **scales)
    o, lse = basp.attn_decode(q[:, 0], *pages, st["lens"], scale=st["scale"],
                              max_len=c["max_len"], **scales)
    return o, lse, st["k_pages"], st["v_pages"]


# ------------------------------------------------------------------- work
def work(case):
    c = case
    size = {"bf16": 2, "f32": 4, "e4m3": 1}
    d = c["d"]
    if c["op"].startswith("norm"):
        tokens, n = c["b"] * c["S"], c["n_q"] + c["n_k"]
        table = c["S"] * c["rot"] * 4
        x = tokens * n * d
        if c["op"] == "norm_rope":
            return {"bytes": x * 2 * size[c["dtype"]] + table + 2 * d * 4, "flops": 8 * x}
        return {"bytes": x * (size[c["dtype"]] + 2 * size[c["grad"]]) + table + 4 * d * 4,
                "flops": 18 * x}
    row = d * size[c["cache"]] + (1 if c["cache"] == "e4m3" else 0)  # a token of a head, with scale
    n_k = c["n_k"]
    if c["op"] == "cache":
        start, count = _starts(c)
        new, old = sum(count), sum(start)
        # new tokens: read, written to the pages, read back; every token's row written out
        return {"bytes": 2 * n_k * (new * (2 * d + 2 * row) + old * row
                                    + c["b"] * (c["ctx"] + c["T"]) * 2 * d),
                "flops": 2 * n_k * (new + old) * d}
    keys = sum(_lens(c))
    got = {"bytes": 2 * n_k * keys * row + c["b"] * c["n_q"] * (d * 4 + 4) + 4 * keys // c["page"],
           "flops": 4.0 * keys * c["n_q"] * d}
    if c["op"] == "step":
        got["bytes"] += c["b"] * (c["n_q"] + n_k) * d * 4 + 4 * c["b"] * n_k * d * 2
    return got


# ------------------------------------------------------------------ exact
def _exact_norm_rope(x, w, cos, sin, rot, interleaved):
    """fp64 from the definition, the rotation as a product of complex numbers."""
    y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
    turn = torch.complex(cos.double(), sin.double())
    head = y[..., :rot]
    if interleaved:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], -1, 2).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(*head.chunk(2, -1)) * turn
        head = torch.cat((z.real, z.imag), -1)
    return torch.cat((head, y[..., rot:]), -1)


def _exact_pow2(e):
    """2^e in fp64 for whole e, from its bits: pow() on the GPU is an ulp off for some."""
    return ((e.long() + 1023) << 52).view(F64)


def _exact_cell(x):
    """The value a row of the 8-bit cache stands for, in fp64: steps of 2^(exponent - 3)."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True) / 448
    e = torch.frexp(top)[1]                         # top in [2^(e-1), 2^e)
    e = torch.where(top == _exact_pow2(e - 1), e - 1, e).clamp(min=E_MIN)
    e = torch.where(top > 0, e, torch.full_like(e, E_MIN))
    u = x * _exact_pow2(-e)
    step = _exact_pow2(torch.frexp(u.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(u / step) * step * _exact_pow2(e)


def _exact_row(st, s, name, n):
    """Sequence s's first n cached tokens, [n_k, n, d] in fp64."""
    pages = st[name + "_pages"]
    page = pages.shape[2]
    at = st["table"][s, :-(-n // page)].long()
    x = pages.view(torch.uint8)[at].view(E4M3).double() if pages.dtype == E4M3 else pages[at].double()
    if pages.dtype == E4M3:
        x = x * _exact_pow2(st[name + "_scales"][at].long()[..., None] - 127)
    return x.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def _exact_attend(q, K, V, scale):
    """q [n_q, d] over K, V [n_k, n, d]: (O [n_q, d], LSE [n_q]) in fp64."""
    n_k, n, d = K.shape
    if n == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=F64, device="cuda")
    s = torch.matmul(q.view(n_k, -1, d), K.transpose(1, 2).contiguous()) * scale
    lse = torch.logsumexp(s, -1)
    return (torch.matmul(torch.exp(s - lse[..., None]), V).reshape(-1, d), lse.reshape(-1))


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"].startswith("norm"):
        x = {n: st[n].double() for n in ("q", "k")}
        w = {n: st[n + "w"].double() for n in ("q", "k")}
        at = slice(c["pos0"], c["pos0"] + c["S"])
        cos, sin = st["cos"][at][:, None], st["sin"][at][:, None]
        if c["op"] == "norm_rope":
            return tuple(_exact_norm_rope(x[n], w[n], cos, sin, c["rot"], c["interleaved"])
                         for n in ("q", "k"))
        got = []
        for n in ("q", "k"):
            a, ww = x[n].requires_grad_(), w[n].requires_grad_()
            y = _exact_norm_rope(a, ww, cos, sin, c["rot"], c["interleaved"])
            got.append(torch.autograd.grad(y, (a, ww), st["d" + n].double()))
        return got[0][0], got[1][0], got[0][1], got[1][1]
    if c["op"] == "cache":
        start, count = _starts(c)
        L = c["ctx"] + c["T"]
        out = []
        for n in ("k", "v"):
            o = torch.zeros(c["b"], L, c["n_k"], c["d"], dtype=F64, device="cuda")
            for s in range(c["b"]):
                o[s, :start[s]] = _exact_row(st, s, n, start[s]).transpose(0, 1)
                new = st[n][s, :count[s]]
                o[s, start[s]:start[s] + count[s]] = (_exact_cell(new) if c["cache"] == "e4m3"
                                                      else new.double())
            out.append(o)
        return tuple(out)
    lens = _lens(c)
    os, lses = [], []
    for s in range(c["b"]):
        K, V = _exact_row(st, s, "k", lens[s]), _exact_row(st, s, "v", lens[s])
        q = st["q"][s].double()
        if c["op"] == "step":
            p = lens[s] - 1
            turn = (st["cos"][p:p + 1][:, None], st["sin"][p:p + 1][:, None], c["d"], False)
            # both are held in bf16 between the operators
            q = _exact_norm_rope(q[None], st["qw"], *turn)[0, 0].to(BF16).double()
            k = _exact_norm_rope(st["k"][s].double()[None], st["kw"], *turn)[0, 0].to(BF16).double()
            K[:, p], V[:, p] = k, st["v"][s, 0].double()
        o, lse = _exact_attend(q, K, V, st["scale"])
        os.append(o)
        lses.append(lse)
    got = torch.stack(os), torch.stack(lses)
    return got if c["op"] == "decode" else (*got, None, None)
