"""The paged key-value cache, and attention of one token over it, against plain fp64."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import F64, check, decode_ref, gather_ref, pow2, quantise_ref

pytestmark = pytest.mark.gpu
BF16, F32, E4M3, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32


def _cache(n_pages, n_k, page, d, e4m3, seed=0):
    """Pages full of NaN: what no call has written must not matter."""
    kw = {}
    if e4m3:
        k = torch.full((n_pages, n_k, page, d), 0x7F, dtype=torch.uint8, device="cuda")
        kw = {n: torch.full((n_pages, n_k, page), 255, dtype=torch.uint8, device="cuda")
              for n in ("k_scales", "v_scales")}
        return k.view(E4M3), k.clone().view(E4M3), kw
    k = torch.full((n_pages, n_k, page, d), math.nan, dtype=BF16, device="cuda")
    return k, k.clone(), kw


def _table(b, max_pages, n_pages, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(n_pages, generator=g)[:b * max_pages].view(b, max_pages).to(I32).cuda()


def _ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def _randn(*s, seed=0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*s, generator=g, device="cuda").to(dtype)


# --------------------------------------------------------------- write, read
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("e4m3", [False, True])
def test_write_and_read(d, page, e4m3):
    b, n_k, T = 5, 3, 45
    start, count = [0, 7, -1, 300, 15], [45, 0, 45, 30, 44]
    mp = -(-400 // page)
    kp, vp, kw = _cache(b * mp + 3, n_k, page, d, e4m3)
    before = [t.clone() for t in (kp.view(torch.uint8), vp.view(torch.uint8), *kw.values())]
    table = _table(b, mp, b * mp + 3)
    k, v = _randn(b, T, n_k, d, seed=1), _randn(b, T, n_k, d, seed=2) * 100
    print("write", d, page, e4m3, flush=True)
    basp.kv_write(k, v, kp, vp, table, _ints(start), count=_ints(count), **kw)
    wrote = torch.zeros(kp.shape[:3], dtype=torch.bool, device="cuda")
    names = ("k_scales", "v_scales")
    held = {n: quantise_ref(x) for n, x in zip(names, (k, v))}
    for s in range(b):
        for t in range(count[s] if start[s] >= 0 else 0):
            p = start[s] + t
            i, r = int(table[s, p // page]), p % page
            wrote[i, :, r] = True
            for x, pages, n in ((k, kp, names[0]), (v, vp, names[1])):
                if e4m3:
                    val, byte = (y[s, t] for y in held[n])
                    assert torch.equal(kw[n][i, :, r], byte)
                    got = pages[i, :, r].double() * pow2(byte.int() - 127)[:, None]
                    assert torch.equal(got, val)
                else:
                    assert torch.equal(pages[i, :, r], x[s, t])
    after = [kp.view(torch.uint8), vp.view(torch.uint8), *kw.values()]
    for x, y in zip(before, after):
        assert torch.equal(x[~wrote], y[~wrote])
    rk, rv = basp.kv_read(kp, vp, table, T, start=_ints(start), count=_ints(count), **kw)
    for s in range(b):
        n = count[s] if start[s] >= 0 else 0
        for x, y in ((k, rk), (v, rv)):
            want = quantise_ref(x[s, :n])[0] if e4m3 else x[s, :n].double()
            assert torch.equal(y[s, :n].double(), want)
            assert (y[s, n:] == 0).all()


def test_every_bf16_value_in_8_bits():
    """Every finite bf16 value beside a row maximum at each distance, the subnormal ones, rows of
    zeros, infinities and NaN."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16)
    fin = bits[bits.isfinite()]
    d = 128
    rows = [fin[: fin.numel() // d * d].view(-1, d)]              # neighbours in magnitude
    g = torch.Generator().manual_seed(3)
    rows.append(fin[torch.randint(0, fin.numel(), (512, d), generator=g)])
    tops = torch.tensor([448., 449., 450., 447., 224., 3.389e38, 1.1755e-38, 2.0 ** -133, 2.0 ** -100,
                         2.0 ** -102 * 1.75, 2.0 ** -102 * 1.7578125, 1.0, 1.75, 1.7578125])
    near = (torch.randn(tops.numel(), d, generator=g).clamp(-0.999, 0.999) * tops[:, None])
    near[:, 5] = tops
    rows.append(near.to(BF16))
    odd = torch.randn(6, d, generator=g)
    odd[0] = 0
    odd[1, 3], odd[2, 4], odd[3, 5] = math.inf, -math.inf, math.nan
    odd[4] = math.inf
    odd[5] = math.nan
    rows.append(odd.to(BF16))
    x = torch.cat(rows).cuda()
    n = x.shape[0]
    mp = -(-n // 256)
    kp, vp, kw = _cache(mp, 1, 256, d, True)
    table = torch.arange(mp, dtype=I32, device="cuda").view(1, -1)
    k = x.view(1, n, 1, d)
    basp.kv_write(k, (-k.float()).to(BF16), kp, vp, table, _ints([0]), **kw)
    want, byte = quantise_ref(x)
    assert torch.equal(kw["k_scales"].view(-1)[:n], byte)
    rk, rv = basp.kv_read(kp, vp, table, n, **kw)
    for y, w in ((rk, want), (rv, -want)):
        y = y.view(n, d).double()
        assert torch.equal(y.isnan(), w.isnan())
        assert torch.equal(y[~y.isnan()], w[~w.isnan()])
    # the bound that the format promises
    live = x.isfinite()
    e = byte.int()[:, None] - 127
    off = (want - x.double()).abs()
    floor = pow2(e - 10).expand_as(off)
    assert (off <= torch.maximum(x.double().abs() * 2.0 ** -4, floor))[live].all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_bad_pages_and_lengths(e4m3):
    """Page numbers out of range, positions past the table: skipped by the write, NaN in the read."""
    b, n_k, page, d, T = 3, 2, 16, 96, 40
    kp, vp, kw = _cache(12, n_k, page, d, e4m3)
    table = torch.arange(9, dtype=I32, device="cuda").view(3, 3).contiguous()
    table[1, 1], table[2, 0] = 12, -5
    before = kp.view(torch.uint8).clone()
    k, v = _randn(b, T, n_k, d, seed=1), _randn(b, T, n_k, d, seed=2)
    start = _ints([20, 0, 0])   # sequence 0 runs past its 48 tokens
    basp.kv_write(k, v, kp, vp, table, start, **kw)
    changed = (before != kp.view(torch.uint8)).flatten(1).any(1)
    assert changed.tolist() == [False, True, True, True, False, True, False, True, True] + [False] * 3
    rk, _ = basp.kv_read(kp, vp, table, T, start=start, **kw)
    nan = rk.isnan().all(-1).all(-1)
    assert nan[0].tolist() == [t >= 28 for t in range(T)]
    assert nan[1].tolist() == [16 <= t < 32 for t in range(T)]
    assert nan[2].tolist() == [t < 16 for t in range(T)]
    assert not rk[~nan].isnan().any()
    top = _ints([2 ** 31 - 1] * 3)
    basp.kv_write(k, v, kp, vp, table, top, **kw)
    rk, rv = basp.kv_read(kp, vp, table, T, start=top, **kw)
    assert rk.isnan().all() and rv.isnan().all()


def test_write_of_strided_tokens():
    b, T, n_q, n_k, d = 2, 9, 4, 2, 80
    qkv = _randn(b, T, n_q + 2 * n_k, d)
    k, v = qkv[:, :, n_q:n_q + n_k], qkv[:, :, n_q + n_k:]
    out = []
    for x, y in ((k, v), (k.contiguous(), v.contiguous())):
        kp, vp, _ = _cache(4, n_k, 16, d, False)
        kp.zero_(), vp.zero_()
        basp.kv_write(x, y, kp, vp, _ints([[2, 0], [3, 1]]), _ints([3, 12]))
        out.append((kp, vp))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


# ------------------------------------------------------------------ attention
def _filled(lens, n_k, page, d, e4m3, spare=2, seed=0, table=None, scale_v=1.0):
    """A cache that holds lens[s] random tokens of each sequence, NaN elsewhere."""
    b, mp = len(lens), max(1, -(-max(lens + [1]) // page))
    kp, vp, kw = _cache(b * mp + spare, n_k, page, d, e4m3)
    table = _table(b, mp, b * mp + spare, seed) if table is None else table
    T = max(lens + [1])
    k, v = _randn(b, T, n_k, d, seed=seed + 1), _randn(b, T, n_k, d, seed=seed + 2) * scale_v
    basp.kv_write(k, v, kp, vp, table, _ints([0] * b), count=_ints(lens), **kw)
    return kp, vp, table, kw


def _check_decode(q, kp, vp, table, lens, kw, scale=None, **more):
    b, n_q, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    print("decode", tuple(q.shape), tuple(kp.shape), kp.dtype, lens[:8], more, flush=True)
    o, lse = basp.attn_decode(q, kp, vp, table, _ints(lens), scale=scale, **kw, **more)
    torch.cuda.synchronize()
    for s in range(b):
        n = max(0, lens[s])
        K = gather_ref(kp, kw.get("k_scales"), table[s], n)
        V = gather_ref(vp, kw.get("v_scales"), table[s], n)
        ro, bo, rl, bl = decode_ref(q[s], K, V, scale)
        check(f"o[{s}]", o[s], ro, bo, BF16)
        check(f"lse[{s}]", lse[s], rl, bl, F32)
    return o, lse


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_q,n_k,page", [(1, 1, 16), (7, 1, 32), (8, 2, 64), (16, 1, 128),
                                          (34, 2, 256), (4, 4, 16)])
def test_decode_heads_and_dims(d, e4m3, n_q, n_k, page):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 200, 257]
    kp, vp, table, kw = _filled(lens, n_k, page, d, e4m3, seed=d)
    _check_decode(_randn(len(lens), n_q, d, seed=9), kp, vp, table, lens, kw)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_q,n_k,L", [(17, 1, 700), (32, 1, 129), (33, 1, 300), (64, 2, 2000),
                                       (80, 1, 1000)])
def test_decode_many_query_heads(d, e4m3, n_q, n_k, L):
    """More than 16 query heads on a kv head: 32 to a workgroup, and several of these."""
    lens = [L, 0, L // 3, 1]
    kp, vp, table, kw = _filled(lens, n_k, 32, d, e4m3, seed=n_q)
    _check_decode(_randn(4, n_q, d, seed=9), kp, vp, table, lens, kw)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("b,L,n_q,n_k,d,page", [
    (1, 1, 8, 1, 128, 64), (1, 5000, 8, 1, 128, 64), (1, 70001, 8, 1, 128, 64),
    (1, 33333, 4, 4, 64, 16), (6, 9001, 7, 1, 80, 32), (2, 20000, 32, 8, 96, 256),
    (300, 130, 2, 1, 64, 16), (64, 3000, 8, 2, 128, 64)])
def test_decode_lengths(e4m3, b, L, n_q, n_k, d, page):
    g = torch.Generator().manual_seed(L)
    lens = [L] + torch.randint(0, L + 1, (b - 1,), generator=g).tolist()
    kp, vp, table, kw = _filled(lens, n_k, page, d, e4m3, seed=L)
    _check_decode(_randn(b, n_q, d, seed=9), kp, vp, table, lens, kw)


@pytest.mark.parametrize("L", list(range(1, 18)) + list(range(30, 35)) + [47, 48, 49, 79, 80, 81, 95,
                                                                          96, 97, 111, 112, 113, 128,
                                                                          129, 255, 256, 511, 512, 513])
@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_every_tail(L, e4m3):
    kp, vp, table, kw = _filled([L], 1, 16, 128, e4m3, seed=L)
    _check_decode(_randn(1, 8, 128, seed=9), kp, vp, table, [L], kw)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_scores_that_rise_fall_and_jump(e4m3):
    """Keys along q with a factor that changes along the sequence: the running maximum moves late,
    early, or by more than fp32's range of exponents at once."""
    d, n, page = 128, 3000, 64
    t = torch.arange(n, device="cuda", dtype=F64)
    shapes = [t / n * 30, (n - t) / n * 30, torch.where(t == 2777, 150.0, -150.0),
              torch.where(t < 1500, -300.0, 0.0), torch.where(t % 64 == 63, 90.0, 0.0),
              torch.where(t == 0, 60.0, 0.0)]
    b = len(shapes)
    q = _randn(b, 8, d, seed=4)
    unit = q[:, :1].double() / q[:, :1].double().pow(2).sum(-1, keepdim=True)
    k = torch.stack([f[:, None, None] * d ** 0.5 * unit[i] for i, f in enumerate(shapes)]).to(BF16)
    v = _randn(b, n, 1, d, seed=5)
    mp = -(-n // page)
    kp, vp, kw = _cache(b * mp, 1, page, d, e4m3)
    table = _table(b, mp, b * mp)
    basp.kv_write(k, v, kp, vp, table, _ints([0] * b), **kw)
    _check_decode(q, kp, vp, table, [n] * b, kw)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_nan_and_infinity(e4m3):
    """A NaN key or value reaches its own sequence and head only; minus infinity as a key's score
    takes its key out; beyond the length nothing matters (the pages are full of NaN there)."""
    lens, n_k, d, page = [300, 300, 300], 2, 64, 32
    kp, vp, table, kw = _filled(lens, n_k, page, d, e4m3)
    q = _randn(3, 4, d, seed=3)
    want, _ = basp.attn_decode(q, kp, vp, table, _ints(lens), **kw)
    kp[int(table[1, 8]), 1, 3, 7] = math.nan
    vp[int(table[2, 2]), 0, 5, 9] = math.nan
    got, lse = basp.attn_decode(q, kp, vp, table, _ints(lens), **kw)
    assert torch.equal(got[0], want[0])
    assert torch.equal(got[1, :2], want[1, :2]) and got[1, 2:].isnan().all()
    assert lse[1, 2:].isnan().all() and not lse[2].isnan().any()
    assert torch.equal(got[2, 2:], want[2, 2:]) and got[2, :2, 9].isnan().all()
    if not e4m3:
        kp, vp, table, kw = _filled([300], 1, page, d, False)
        q = _randn(1, 2, d, seed=3).abs()
        kp[int(table[0, 0]), 0, 3] = -math.inf
        kp[int(table[0, 9]), 0, 11] = -math.inf   # the last token: position 299
        K, V = gather_ref(kp, None, table[0], 300), gather_ref(vp, None, table[0], 300)
        keep = [i for i in range(300) if i not in (3, 299)]
        o, lse = basp.attn_decode(q, kp, vp, table, _ints([300]))
        ro, bo, rl, bl = decode_ref(q[0], K[keep].contiguous(), V[keep].contiguous(), d ** -0.5)
        check("o", o[0], ro, bo, BF16)
        check("lse", lse[0], rl, bl, F32)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_decode_keys_of_minus_infinity(d):
    """A key whose first, or last, elements are minus infinity against a positive query is taken
    out: its score is minus infinity, whatever the row's padding to whole operands reads."""
    kp, vp, table, _ = _filled([150], 1, 16, d, False)
    q = _randn(1, 3, d, seed=3).abs() + 0.5
    out = (3, 40, 149)
    for i, t in enumerate(out):
        col = slice(0, 8) if i % 2 else slice(d - 4, d)
        kp[int(table[0, t // 16]), 0, t % 16, col] = -math.inf
    K, V = gather_ref(kp, None, table[0], 150), gather_ref(vp, None, table[0], 150)
    keep = [i for i in range(150) if i not in out]
    o, lse = basp.attn_decode(q, kp, vp, table, _ints([150]))
    ro, bo, rl, bl = decode_ref(q[0], K[keep].contiguous(), V[keep].contiguous(), d ** -0.5)
    check("o", o[0], ro, bo, BF16)
    check("lse", lse[0], rl, bl, F32)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_bad_pages_and_lengths(e4m3):
    lens = [100, 100, 100, 40, 200, -7]
    kp, vp, table, kw = _filled([100, 100, 100, 40, 100, 0], 1, 16, 128, e4m3)
    q = _randn(6, 8, 128, seed=3)
    table[1, 6] = table[3, 5] = kp.shape[0]   # page 5 of sequence 3 lies past its 40 tokens
    table[2, 0] = -1
    o, lse = basp.attn_decode(q, kp, vp, table, _ints(lens), **kw)  # the table holds 112 tokens
    for s in range(6):
        if s in (1, 2, 4):
            assert o[s].isnan().all() and lse[s].isnan().all(), s
        else:
            assert not o[s].isnan().any(), s
    assert (o[5] == 0).all() and (lse[5] == -math.inf).all()
    o, lse = basp.attn_decode(q[:1], kp, vp, table[:1], _ints([100]), max_len=99, **kw)
    assert o.isnan().all() and lse.isnan().all()
    _check_decode(q[:1], kp, vp, table[:1].contiguous(), [100], kw, max_len=100)
    _check_decode(q[:1], kp, vp, table[:1].contiguous(), [100], kw, max_len=100000)


def test_decode_shared_pages_strides_and_scale():
    """Two sequences on the same pages, q as columns of a wider tensor, another scale, no workspace
    reuse between calls of other sizes; the same bits twice, whatever the workspace holds."""
    lens = [900, 900, 500]
    kp, vp, table, kw = _filled(lens, 2, 64, 96, False)
    table[1, :14] = table[0, :14]
    qkv = _randn(3, 1, 8 + 4, 96, seed=3)
    q = qkv[:, 0, :8]
    assert not q.is_contiguous()
    o, lse = _check_decode(q, kp, vp, table, lens, kw, scale=0.3)
    need = basp.attn_decode_workspace_bytes(3, 8, 2, 96, 960)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    o2, lse2 = basp.attn_decode(q.contiguous(), kp, vp, table, _ints(lens), scale=0.3, workspace=ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_cache_beyond_32_bit_offsets():
    """Pages past 4 GiB of a pool, in both types."""
    for e4m3 in (False, True):
        page, d = 256, 128
        n_pages = (2 ** 32 // (page * d * (1 if e4m3 else 2))) + 40
        dt = torch.uint8 if e4m3 else BF16
        kp, vp = (torch.empty(n_pages, 1, page, d, dtype=dt, device="cuda") for _ in range(2))
        kw = {}
        if e4m3:
            kp, vp = kp.view(E4M3), vp.view(E4M3)
            kw = {n: torch.empty(n_pages, 1, page, dtype=torch.uint8, device="cuda")
                  for n in ("k_scales", "v_scales")}
        table = _ints([[n_pages - 1, 3, n_pages - 7], [0, n_pages - 2, 1]])
        k, v = _randn(2, 700, 1, d, seed=1), _randn(2, 700, 1, d, seed=2)
        basp.kv_write(k, v, kp, vp, table, _ints([0, 0]), **kw)
        rk, rv = basp.kv_read(kp, vp, table, 700, **kw)
        want = quantise_ref(k)[0] if e4m3 else k.double()
        assert torch.equal(rk.double(), want)
        _check_decode(_randn(2, 8, d, seed=3), kp, vp, table, [700, 699], kw)
        del kp, vp, kw
        torch.cuda.empty_cache()


def test_cache_empty():
    kp, vp, _ = _cache(2, 1, 16, 64, False)
    z = torch.zeros(0, dtype=I32, device="cuda")
    basp.kv_write(_randn(0, 3, 1, 64), _randn(0, 3, 1, 64), kp, vp, z.view(0, 2), z)
    basp.kv_write(_randn(1, 0, 1, 64), _randn(1, 0, 1, 64), kp, vp, _ints([[0, 1]]), _ints([0]))
    k, v = basp.kv_read(kp, vp, _ints([[0, 1]]), 0)
    assert k.shape == (1, 0, 1, 64)
    o, lse = basp.attn_decode(_randn(0, 2, 64), kp, vp, z.view(0, 2), z)
    assert o.shape == (0, 2, 64) and lse.shape == (0, 2) and kp.isnan().all()


# ------------------------------------------------------------ together
def _step(q, k, v, w, cos, sin, kp, vp, table, lens, kw, ws=None):
    """One token per sequence: norm and rotation, write, attention.  A length of 0: a padded slot."""
    pos = lens - 1
    q, k = basp.qk_norm_rope(q, k, *w, cos, sin, positions=pos.view(-1, 1))
    basp.kv_write(k, v, kp, vp, table, pos, **kw)
    return basp.attn_decode(q[:, 0], kp, vp, table, lens, workspace=ws, **kw)


@pytest.mark.parametrize("e4m3", [False, True])
def test_generation_after_a_prompt(e4m3):
    """A prompt by the share's attention over the whole sequence, its K and V into the cache, then
    token by token: in bf16 every step is the last row of attention over the longer sequence."""
    b, S, n_q, n_k, d, page, new = 2, 300, 8, 2, 128, 64, 5
    L = S + new
    x = [_randn(b, L, n, d, seed=i) for i, n in enumerate((n_q, n_k, n_k))]
    w = 1 + 0.2 * _randn(d, seed=7, dtype=F32), 1 + 0.2 * _randn(d, seed=8, dtype=F32)
    cos, sin = basp.rope_table(L, d)
    Q, K = basp.qk_norm_rope(x[0], x[1], *w, cos, sin)
    mp = -(-L // page)
    kp, vp, kw = _cache(b * mp, n_k, page, d, e4m3)
    table = _table(b, mp, b * mp)
    basp.kv_write(K[:, :S].contiguous(), x[2][:, :S].contiguous(), kp, vp, table, _ints([0] * b), **kw)
    for t in range(S, L):
        row = [y[:, t:t + 1].contiguous() for y in x]
        o, lse = _step(*row, w, cos, sin, kp, vp, table, _ints([t + 1] * b), kw)
        for s in range(b):
            Kc = gather_ref(kp, kw.get("k_scales"), table[s], t + 1)
            Vc = gather_ref(vp, kw.get("v_scales"), table[s], t + 1)
            if not e4m3:  # the cache holds what attention over the whole sequence sees
                assert torch.equal(Kc, K[s, :t + 1].double())
                assert torch.equal(Vc, x[2][s, :t + 1].double())
            ro, bo, rl, bl = decode_ref(Q[s, t], Kc, Vc, d ** -0.5)
            check("o", o[s], ro, bo, BF16)
            check("lse", lse[s], rl, bl, F32)
    if not e4m3:
        O, LSE = basp.attn_fwd(Q, K, x[2])
        ro, bo, _, bl = decode_ref(Q[0, L - 1], K[0].double(), x[2][0].double(), d ** -0.5)
        # both round their weights and results: twice the bound, two last roundings
        assert ((o[0].double() - O[0, L - 1].double()).abs() <= 2 * bo + 2 ** -7 * ro.abs()).all()
        assert ((lse[0] - LSE[0, :, L - 1]).abs() <= 2 * bl + 2 ** -10).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_captured_steps(e4m3):
    """Two graphs of a step (a batch of 4 with a padded slot, a batch of 2), a workspace each,
    replayed in turn with eager work between, against eager steps on a copy of the cache."""
    n_q, n_k, d, page, mp = 8, 2, 128, 16, 8
    kp, vp, kw = _cache(4 * mp, n_k, page, d, e4m3)
    table = _table(4, mp, 4 * mp)
    cos, sin = basp.rope_table(mp * page, d)
    w = 1 + 0.2 * _randn(d, seed=7, dtype=F32), 1 + 0.2 * _randn(d, seed=8, dtype=F32)
    prompt = _randn(4, 60, n_k, d, seed=1), _randn(4, 60, n_k, d, seed=2)
    basp.kv_write(*prompt, kp, vp, table, _ints([0] * 4), **kw)
    kp2, vp2 = kp.clone(), vp.clone()
    kw2 = {n: t.clone() for n, t in kw.items()}
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    runs = []
    for b in (4, 2):
        bufs = [torch.zeros(b, 1, n, d, dtype=BF16, device="cuda") for n in (n_q, n_k, n_k)]
        lens = torch.zeros(b, dtype=I32, device="cuda")
        tab = table[:b].contiguous()
        ws = torch.empty(max(16, basp.attn_decode_workspace_bytes(b, n_q, n_k, d, mp * page)),
                         dtype=torch.uint8, device="cuda")
        with torch.cuda.stream(st):
            _step(*bufs, w, cos, sin, kp, vp, tab, lens, kw, ws)   # all slots padded: writes nothing
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                out = _step(*bufs, w, cos, sin, kp, vp, tab, lens, kw, ws)
        runs.append((graph, bufs, lens, tab, out))
    now = [60, 60, 60, 60]
    for i in range(6):
        graph, bufs, lens, tab, out = runs[i % 2]
        b = lens.numel()
        here = [n + 1 for n in now[:b]]
        if b == 4:
            here[2] = 0
        for j, t in enumerate(bufs):
            t.copy_(_randn(*t.shape, seed=100 * i + j))
        lens.copy_(_ints(here))
        graph.replay()
        torch.cuda.synchronize()
        want = _step(*bufs, w, cos, sin, kp2, vp2, tab, _ints(here), kw2)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), i
        assert torch.equal(kp.view(torch.uint8), kp2.view(torch.uint8)), i
        for s, n in enumerate(here):
            now[s] = n if n else now[s]


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("b,n_q,L", [(1, 8, 3000), (7, 5, 300), (40, 20, 500)])
def test_decode_and_read_write_nothing_else(d, e4m3, b, n_q, L):
    """Outputs and workspace inside larger buffers: what lies around them stays, and a workspace of the
    size reported is enough."""
    lens = [L] + [(37 * i) % L for i in range(1, b)]
    kp, vp, table, kw = _filled(lens, 1, 32, d, e4m3)

    def inside(dtype, shape):
        n = math.prod(shape)
        buf = torch.full((n + 128,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[64:64 + n].view(shape)

    need = basp.attn_decode_workspace_bytes(b, n_q, 1, d, L)
    assert need % 4 == 0
    ob, o = inside(BF16, (b, n_q, d))
    lb, lse = inside(F32, (b, n_q))
    wb, ws = inside(F32, (need // 4,))
    kb, k = inside(BF16, (b, 33, 1, d))
    vb, v = inside(BF16, (b, 33, 1, d))
    q = _randn(b, n_q, d, seed=3)
    basp.attn_decode(q, kp, vp, table, _ints(lens), max_len=L, out=o, lse=lse, workspace=ws, **kw)
    basp.kv_read(kp, vp, table, 33, count=_ints([min(33, n) for n in lens]), k=k, v=v, **kw)
    for buf in (ob, lb, wb, kb, vb):
        assert (buf[:64] == 7).all() and (buf[-64:] == 7).all()
    ro, rl = basp.attn_decode(q, kp, vp, table, _ints(lens), max_len=L, **kw)
    assert torch.equal(o, ro) and torch.equal(lse, rl)
