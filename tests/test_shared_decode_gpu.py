"""attn_decode_shared: one new token for sequences that share prefixes, against plain fp64."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import F64, TINY, U16, U32, check, gather_ref
from paper_2609_03151_amd.cache import PagedKV

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731


def _slopes(n):
    return 2.0 ** (-8.0 * torch.arange(1, n + 1, dtype=F32, device="cuda") / n)


class Case:
    """Pages, table and lengths: sizes[g] sequences in group g, prefix[g] tokens, own[s] tokens
    past it (negative: the sequence ends inside the prefix, or has no keys)."""

    def __init__(self, sizes, prefix, own, n_q, n_k, d, page, dtype, seed=0, spare=2, fill=0.0):
        g = torch.Generator("cuda").manual_seed(seed)
        b = sum(sizes)
        first = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
        of = [i for i, n in enumerate(sizes) for _ in range(n)]
        self.lens_list = [max(0, prefix[of[s]] + own[s]) for s in range(b)]
        self.max_len = max(max(self.lens_list), 1)
        mp = -(-self.max_len // page) + 1
        table = torch.full((b, mp), -1, dtype=torch.int64)
        n, copies = spare, []
        for i, p in enumerate(prefix):
            whole, own_first = p // page, None
            shared = torch.arange(n, n + whole)
            n += whole
            for s in range(first[i], first[i + 1]):
                table[s, :whole] = shared[:mp]
                more = -(-self.lens_list[s] // page) - whole
                if more > 0:
                    table[s, whole:whole + more] = torch.arange(n, n + more)
                    if p % page:
                        if own_first is None:
                            own_first = n
                        else:
                            copies.append((n, own_first, p % page))
                    n += more
        order = torch.randperm(n, generator=g, device="cuda")
        self.table = torch.where(table.cuda() < 0, table.cuda(), order[table.cuda().clamp(min=0)]
                                 ).to(torch.int32)
        self.cache = PagedKV(n, n_k, d, page=page, dtype=dtype)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        for name in ("k", "v"):
            pages = getattr(self.cache, name + "_pages")
            if dtype == E4M3:
                bits = torch.randint(0, 256, pages.shape, generator=g, device="cuda")
                bits = torch.where(bits % 128 == 127, 0, bits).to(torch.uint8)
                pages.view(torch.uint8).copy_(bits)
                scales = getattr(self.cache, name + "_scales")
                scales.copy_(torch.randint(119, 122, scales.shape, generator=g, device="cuda"))
            else:
                pages.copy_(rn(*pages.shape))
            for to, frm, m in copies:
                pages.view(torch.uint8 if dtype == E4M3 else torch.int16)[order[to], :, :m] = \
                    pages.view(torch.uint8 if dtype == E4M3 else torch.int16)[order[frm], :, :m]
                if dtype == E4M3:
                    scales[order[to], :, :m] = scales[order[frm], :, :m]
        self.q = (2 * rn(b, n_q, d)).to(BF16)
        self.lens, self.groups, self.prefix = ints(self.lens_list), ints(first), ints(prefix)
        self.b, self.n_q, self.n_k, self.d = b, n_q, n_k, d

    def run(self, cap=None, slopes=None, groups=True, **more):
        return self.cache.attend_shared(self.q, self.table, self.lens,
                                        self.groups if groups else None,
                                        self.prefix if groups else None, scale=0.1,
                                        max_len=self.max_len, cap=cap, slopes=slopes, **more)

    def ref(self, s, cap, slopes):
        """(O, bound, LSE, bound) of sequence s, as span_ref's."""
        c, n = self.cache, self.lens_list[s]
        if n == 0:
            z = torch.zeros(self.n_q, self.d, dtype=F64, device="cuda")
            l = torch.full((self.n_q,), -math.inf, dtype=F64, device="cuda")
            return z, z, l, torch.zeros_like(l)
        K = gather_ref(c.k_pages, c.k_scales, self.table[s], n)
        V = gather_ref(c.v_pages, c.v_scales, self.table[s], n)
        rep = self.n_q // self.n_k
        Q = self.q[s].double().view(self.n_k, rep, self.d)
        Kt = K.permute(1, 2, 0).contiguous()
        u = torch.matmul(Q, Kt).view(self.n_q, n) * 0.1
        e = torch.matmul(Q.abs(), Kt.abs()).view(self.n_q, n) * 0.1 * (self.d + 16) * U32
        if cap:
            t = torch.tanh(u / cap)
            e = e * (1 - t * t) + cap * (2.0 ** -21 + 2 * U32) + e * e / cap
            u = cap * t
        e = e + 6 * U32 * u.abs()
        if slopes is not None:
            bias = slopes.double()[:, None] * (n - 1 - torch.arange(n, device="cuda"))
            u, e = u - bias, e + 6 * U32 * bias.abs()
        lse = torch.logsumexp(u, -1)
        p = torch.exp(u - lse[:, None])
        Vh = V.transpose(0, 1).contiguous()
        heads = lambda w: torch.matmul(w.view(self.n_k, rep, n), Vh)  # noqa: E731
        mags = lambda w: torch.matmul(w.view(self.n_k, rep, n), Vh.abs())  # noqa: E731
        O = heads(p).view(self.n_q, self.d)
        worst = e.amax(-1, keepdim=True)
        # weights rounded to bf16 once, their exponents, the row's sum, fp32 sums and the join's
        # weights of partial results (some 2^-20 each); weights below 2^-126 of a partial result
        bound = mags(p * (U16 + 2.0 ** -17 + (2 * n + 64) * U32 + e + worst))
        bound = (bound + mags(torch.full_like(p, 2.0 ** -33))).view(self.n_q, self.d) * 1.01
        el = worst[:, 0] + 2.0 ** -18 + (n + 16) * U32 + 4 * U32 * (lse.abs() + u.abs().amax(-1))
        return O, bound + TINY, lse, el

    def check(self, cap=None, slopes=None, **more):
        print(f"case {tuple(self.q.shape)} {tuple(self.cache.k_pages.shape)} lens {self.lens_list[:8]} "
              f"cap {cap} slopes {slopes is not None}", flush=True)
        o, lse = self.run(cap, slopes, **more)
        assert o.dtype == BF16 and lse.dtype == F32
        refs = [self.ref(s, cap, slopes) for s in range(self.b)]
        check("o", o, torch.stack([r[0] for r in refs]), torch.stack([r[1] for r in refs]), BF16)
        check("lse", lse, torch.stack([r[2] for r in refs]), torch.stack([r[3] for r in refs]), F32)
        return o, lse


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("rule", ["plain", "cap", "large cap", "bias", "both"])
def test_dims_and_rules(d, dtype, rule):
    c = Case([3, 1, 4], [300, 50, 129], [40, 1, 200, 33, 5, 0, -20, 129], 8, 2, d, 32, dtype, seed=d)
    cap = {"cap": 10.0, "both": 30.0, "large cap": 200.0}.get(rule)
    c.check(cap, _slopes(8) if rule in ("bias", "both") else None)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n_q,n_k", [(1, 1), (7, 1), (8, 8), (16, 1), (40, 2), (34, 1)])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_heads_and_pages(page, n_q, n_k, dtype):
    c = Case([5, 2], [513, 64], [1, 1, 300, -513, 17, 1000, 2], n_q, n_k, 128, page, dtype, seed=n_q)
    c.check()
    c.check(cap=20.0, slopes=_slopes(n_q))


@pytest.mark.parametrize("sizes,prefix,own", [
    ([1], [0], [1]), ([1], [0], [77]), ([2], [1], [0, 0]), ([2], [1], [1, 0]), ([2], [16], [0, 0]),
    ([2], [63], [1, 2]), ([3], [64], [0, 1, -1]), ([2], [65], [1, 1]), ([2, 2], [0, 0], [1, 5, 3, 2]),
    ([4], [1000], [-1000, -999, -1, 0]), ([2], [4000], [-4000, -4000]), ([70], [130], list(range(70))),
    ([1, 1, 1, 1], [500, 400, 300, 200], [1, 2, 3, 4]), ([16, 17, 31], [2049, 777, 48], [3] * 64),
    ([3], [9000], [128, 129, 3000]), ([129], [31], [0] * 129),
])
@pytest.mark.parametrize("bias", [False, True])
def test_groups_and_lengths(sizes, prefix, own, bias):
    c = Case(sizes, prefix, own, 4, 1, 64, 16, BF16, seed=len(own))
    c.check(slopes=_slopes(4) if bias else None)


def test_many_sequences():
    """More sequences than a workgroup's threads, and than are searched side by side; more groups
    than a workgroup has waves."""
    for b, per in ((1100, 11), (2200, 2)):
        own = [(7 * s) % 60 - 5 for s in range(b)]
        c = Case([per] * (b // per), [20 + g % 50 for g in range(b // per)], own, 2, 1, 64, 16, BF16,
                 seed=b)
        c.check(cap=30.0)


def test_slopes_of_any_sign():
    c = Case([4, 3], [700, 90], [5, 100, 1, 0, 3, 2, 400], 4, 2, 128, 64, BF16, seed=4)
    for slopes in ([-0.05, 0.0, 40.0, 0.5], [-1.0, -0.001, 3.0, 100.0]):
        for cap in (None, 12.0, 500.0):
            c.check(cap, torch.tensor(slopes, device="cuda"))


def test_without_groups_is_attn_decode():
    """Nothing shared, no rule: to the roundings of the weights what attn_decode gives; and with the
    prefix shared too."""
    c = Case([6], [1500], [1, 700, 30, 0, 2, 9], 8, 2, 128, 64, E4M3, seed=1)
    want, lse = c.cache.attend(c.q, c.table, c.lens, scale=0.1, max_len=c.max_len)
    for groups in (False, True):
        o, l = c.check(groups=groups) if groups else c.run(groups=False)
        bound = torch.stack([c.ref(s, None, None)[1] for s in range(c.b)])
        assert ((o.double() - want.double()).abs() <= 2 * bound + 2.0 ** -7 * want.double().abs()).all()
        assert (l - lse).abs().max() <= 1e-4


def test_garbage_where_nobody_looks():
    """Pages past the lengths, of dead slots and not in any row hold NaN; dead slots' rows of the
    table any numbers, a group's first slot among them."""
    c = Case([4, 3], [100, 40], [-100, 30, 1, 0, 5, -40, 64], 4, 2, 128, 32, BF16, seed=9)
    used = torch.zeros(c.cache.k_pages.shape[0], 32, dtype=torch.bool, device="cuda")
    for s, n in enumerate(c.lens_list):
        for t in range(n):
            used[c.table[s, t // 32], t % 32] = True
    want = c.check()
    for pages in (c.cache.k_pages, c.cache.v_pages):
        pages.copy_(torch.where(used[:, None, :, None], pages, math.nan))
    c.table[0] = 2 ** 31 - 1
    c.table[5] = -7
    got = c.run()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_bad_pages_and_lengths(dtype):
    """A page number out of range makes NaN of the sequences that reach it, a length past the
    largest of its own; the others' results stay."""
    c = Case([3, 2], [200, 64], [10, 70, 1, 3, 90], 4, 1, 96, 16, dtype, seed=2)
    o, lse = c.run()
    table = c.table.clone()
    c.table[1, 201 // 16] = c.cache.k_pages.shape[0]      # an own page
    o2, lse2 = c.run()
    live = [0, 2, 3, 4]
    assert o2[1].isnan().all() and lse2[1].isnan().all()
    assert torch.equal(o2[live], o[live]) and torch.equal(lse2[live], lse[live])
    c.table.copy_(table)
    c.table[0, 3] = -1                                     # a page of the prefix, in its first row
    o2, lse2 = c.run()
    assert o2[:3].isnan().all() and lse2[:3].isnan().all() and torch.equal(o2[3:], o[3:])
    c.table.copy_(table)
    c.lens[0] = c.max_len + 1                              # shares nothing any more
    o2, lse2 = c.run()
    assert o2[0].isnan().all() and torch.equal(lse2[1:], lse[1:])
    c.lens[0] = -5
    o2, lse2 = c.run()
    assert (o2[0] == 0).all() and (lse2[0] == -math.inf).all() and torch.equal(o2[1:], o[1:])
    # the table holds fewer tokens than the lengths say
    c.lens.copy_(ints(c.lens_list))
    c.max_len = 10 ** 6
    c.lens[4] = c.table.shape[1] * 16 + 1
    assert c.run()[0][4].isnan().all()


def test_values_that_are_not_finite():
    """A value of the prefix makes its element NaN or infinite for all who see it, nothing else."""
    c = Case([4], [300], [10, 0, -1, 70], 4, 2, 64, 16, BF16, seed=5)
    o, _ = c.run()
    c.cache.v_pages[c.table[0, 2], 1, 5, 11] = math.inf
    o2, _ = c.run()
    bad = torch.zeros_like(o, dtype=torch.bool)
    bad[:, 2:, 11] = True
    assert not o2[bad].isfinite().any() and torch.equal(o2[~bad], o[~bad])


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("prefix", [1, 20, 40, 300, 331])
def test_keys_past_a_prefix(prefix, dtype):
    """Whatever lies in pages of nobody, the first among them; and an infinite value at a prefix's
    last key, which is read again for the keys past it, reaches its element alone."""
    c = Case([4], [prefix], [10, 0, -1, 70], 4, 2, 64, 16, dtype, seed=prefix)
    names = c.table[c.table >= 0]
    free = next(p for p in range(c.cache.k_pages.shape[0]) if not (names == p).any())
    pools = [c.cache.k_pages, c.cache.v_pages]
    pools += [c.cache.k_scales, c.cache.v_scales] if dtype == E4M3 else []
    for pool in pools:
        raw = pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)
        raw[free] = raw[0]
    c.table.copy_(torch.where(c.table == 0, free, c.table))
    for pool in pools:
        raw = pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)
        raw[0] = 0x7F if pool.element_size() == 1 else 0x7FC0
    c.check()
    if dtype == E4M3:
        return
    t = prefix - 1
    for s in (0, 1, 3):  # 2 ends before it
        c.cache.v_pages[c.table[s, t // 16], 1, t % 16, 11] = math.inf
    o, _ = c.run()
    assert not o[[0, 1, 3], 2:, 11].isfinite().any()
    assert o[2].isfinite().all() and o[:, :, :11].isfinite().all() and o[:, :2].isfinite().all()
    assert o[:, :, 12:].isfinite().all()


def test_group_ends_out_of_range():
    """Ends before the first sequence and past the last are taken for these."""
    c = Case([3, 4], [200, 100], [1, 2, 3, 4, 5, 6, 7], 4, 1, 64, 16, BF16, seed=6)
    want = c.run()
    c.groups.copy_(ints([-(2 ** 31), 3, 2 ** 31 - 1]))
    for x, y in zip(c.run(), want):
        assert torch.equal(x, y)
    # negative prefixes, and ones nobody reaches: nothing is shared
    plain = c.run(groups=False)
    c.prefix.copy_(ints([-3, 2 ** 31 - 1]))
    for x, y in zip(c.run(), plain):
        assert torch.equal(x, y)


@pytest.mark.parametrize("per,b", [(4, 8), (300, 600)])
def test_groups_out_of_order(per, b):
    """Ends that do not ascend: other results, nothing outside the buffers, nothing left behind."""
    g = b // per
    c = Case([per] * g, [50] * g, [s % 7 for s in range(b)], 2, 1, 64, 16, BF16, seed=b)
    want = c.run()
    good = c.groups.clone()
    need = basp.attn_decode_shared_workspace_bytes(b, 2, 1, 64, c.max_len, g)
    ws = torch.full((need + 512,), 255, device="cuda", dtype=torch.uint8)
    for ends in ([b, 0, per], [0, b, per], [per, 2 * per, 0], [0, b, b], [0, 0, per]):
        c.groups.copy_(ints(ends))
        c.run(workspace=ws[256:256 + need])
        assert (ws[:256] == 255).all() and (ws[-256:] == 255).all()
    c.groups.copy_(good)
    for x, y in zip(c.run(workspace=ws[256:256 + need]), want):
        assert torch.equal(x, y)


def test_strides_streams_and_buffers():
    """Q as columns of a wider tensor; outputs and the workspace inside larger buffers; another
    stream; the same bits each time."""
    c = Case([5, 3], [1000, 300], [100] * 8, 8, 2, 128, 64, BF16, seed=7)
    want = c.run(cap=30.0)
    wide = torch.randn(8, 12, 128, device="cuda").to(BF16)
    wide[:, :8] = c.q
    narrow, c.q = c.q, wide[:, :8]
    need = basp.attn_decode_shared_workspace_bytes(8, 8, 2, 128, c.max_len, 2)
    ws = torch.full((need + 512,), 255, device="cuda", dtype=torch.uint8)
    buf = torch.full((8 * 8 * 128 + 128,), 7.0, device="cuda", dtype=BF16)
    out = buf[64:-64].view(8, 8, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            got = c.run(cap=30.0, out=out, workspace=ws[256:256 + need])
            side.synchronize()
            for x, y in zip(got, want):
                assert torch.equal(x, y)
    assert (ws[:256] == 255).all() and (ws[-256:] == 255).all()
    assert (buf[:64] == 7).all() and (buf[-64:] == 7).all()


def test_graph():
    """Captured; replays after new lengths, prefixes, pages and queries equal eager calls."""
    c = Case([5, 3], [1000, 300], [100, 3, 200, 1, 0, 9, 30, 77], 8, 2, 128, 64, E4M3, seed=8)
    ws = torch.empty(basp.attn_decode_shared_workspace_bytes(8, 8, 2, 128, c.max_len, 2),
                     device="cuda", dtype=torch.uint8)
    c.run(workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.run(cap=20.0, slopes=None, workspace=ws)
    for lens, prefix in (([1100, 0, 1000, 1001, 50, 300, 301, 1], [1000, 300]),
                         ([64, 64, 0, 64, 100, 20, 310, 299], [64, 20]),
                         ([1200] * 8, [0, 0])):
        c.lens.copy_(ints(lens))
        c.prefix.copy_(ints(prefix))
        c.q.copy_(torch.randn(c.q.shape, device="cuda"))
        c.lens_list = lens
        c.table.copy_(torch.randint(0, c.cache.k_pages.shape[0], c.table.shape, device="cuda"))
        c.table[1:5] = c.table[0]
        c.table[6:] = c.table[5]
        want = [x.clone() for x in c.run(cap=20.0)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, want):
            assert torch.equal(x, y)
        c.check(cap=20.0)


def test_empty():
    c = Case([1], [0], [1], 4, 2, 64, 16, BF16)
    o, lse = basp.attn_decode_shared(c.q[:0], c.cache.k_pages, c.cache.v_pages, c.table[:0],
                                     c.lens[:0], ints([0]), ints([]))
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
    c.check(groups=False)
    o, _ = c.cache.attend_shared(c.q, c.table, c.lens, ints([0]), ints([]), scale=0.1)
    assert torch.equal(o, c.run(groups=False)[0])


def test_pools_past_4_gib():
    """Pages all over pools of 5 GB each."""
    c = Case([5, 3], [1000, 300], [100, 3, 200, 1, 0, 9, 30, 77], 8, 2, 128, 64, BF16, seed=10,
             spare=160000)
    assert c.cache.k_pages.numel() * 2 > 2 ** 32
    assert c.table.max() * 2 * 64 * 128 * 2 > 2 ** 32
    c.check(cap=20.0, slopes=_slopes(8))


@pytest.mark.parametrize("groups", [2, 300])
def test_two_calls_at_once(groups):
    """Calls on two streams side by side, a workspace each, one of them a graph's: the bits of one
    after the other."""
    cases = [Case([3] * groups, [200] * groups, [i + s % 40 for s in range(3 * groups)], 4, 2, 64, 16,
                  BF16, seed=i) for i in (1, 2)]
    want = [[x.clone() for x in c.run(cap=9.0)] for c in cases]
    spaces = [torch.empty(basp.attn_decode_shared_workspace_bytes(c.b, 4, 2, 64, c.max_len, groups),
                          device="cuda", dtype=torch.uint8) for c in cases]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cases[1].run(cap=9.0, workspace=spaces[1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[1]):
            graph.replay()
        with torch.cuda.stream(streams[0]):
            got = cases[0].run(cap=9.0, workspace=spaces[0])
        torch.cuda.synchronize()
        for x, y in zip((*got, *out), (*want[0], *want[1])):
            assert torch.equal(x, y)
