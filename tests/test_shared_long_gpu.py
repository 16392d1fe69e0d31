"""attn_decode_shared on sequences of more than 2^24 tokens, whose positions fp32 no longer holds."""
import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import TINY, U16, U32, check, gather_ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("cap", [None, 20.0])
@pytest.mark.parametrize("length", [(1 << 24) + 12345, (1 << 25) + 77])
def test_bias_of_the_nearest_keys(shared, cap, length):
    """Slopes that leave the last keys most of the weight: distances are exact there.  The same few pages
    over and over; the reference takes the last 1024 keys, the others weigh less than 2^-140."""
    d, n_q, n_k, page, b, near = 64, 4, 1, 256, 3, 1024
    g = torch.Generator("cuda").manual_seed(length)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    k, v, q = rn(24, n_k, page, d), rn(24, n_k, page, d), rn(b, n_q, d)
    lens = [length, length + 9, length - 300]
    max_pages = -(-max(lens) // page)
    row = torch.randint(0, 24, (max_pages,), generator=g, device="cuda")
    table = row.expand(b, max_pages).to(torch.int32).contiguous()
    slopes = torch.tensor([0.125, 0.25, 0.5, 2.0], device="cuda")
    more = dict(groups=ints([0, 3]), prefix_lens=ints([length - 300])) if shared else {}
    print(f"case {length} {shared} {cap}", flush=True)
    o, lse = basp.attn_decode_shared(q, k, v, table, ints(lens), scale=0.1, cap=cap, slopes=slopes,
                                     **more)
    for s, n in enumerate(lens):
        first = (n - near) // page * page
        cut = table[s, first // page:].contiguous()
        K = gather_ref(k, None, cut, n - first)[:, 0]
        V = gather_ref(v, None, cut, n - first)[:, 0]
        Q = q[s].double()
        u = torch.mm(Q, K.t().contiguous()) * 0.1
        e = torch.mm(Q.abs(), K.abs().t().contiguous()) * 0.1 * (d + 16) * U32
        if cap:
            e = e + cap * (2.0 ** -21 + 2 * U32) + e * e / cap
            u = cap * torch.tanh(u / cap)
        bias = slopes.double()[:, None] * (n - 1 - first - torch.arange(n - first, device="cuda"))
        u, e = u - bias, e + 6 * U32 * (u.abs() + bias)
        L = torch.logsumexp(u, 1)
        p = torch.exp(u - L[:, None])
        O = torch.mm(p, V)
        # as test_shared_decode_gpu's: weights rounded once, their exponents, fp32 sums (here of up to
        # 2^25 terms, 128 at a time over many workgroups: those far away are 0)
        bound = torch.mm(p * (U16 + 2.0 ** -16 + 2 * e.amax(1, keepdim=True)), V.abs()) * 1.01
        check(f"o {s}", o[s], O, bound + TINY, BF16)
        check(f"lse {s}", lse[s], L, e.amax(1) + 2.0 ** -16 + 8 * U32 * L.abs(), F32)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("length", [1, 17, 64, 200, 321])
def test_steep_slopes(shared, length):
    """Slopes that leave the nearest key alone: O is its V, the LSE its score, without the rounding of
    any farther key's bias."""
    d, n_q, n_k, page, b = 128, 4, 2, 16, 2
    g = torch.Generator("cuda").manual_seed(length)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    max_pages = -(-length // page)
    k, v, q = rn(max_pages, n_k, page, d), rn(max_pages, n_k, page, d), rn(b, n_q, d)
    table = torch.arange(max_pages, dtype=torch.int32, device="cuda").expand(b, -1).contiguous()
    slopes = 2.0 ** torch.tensor([10.0, 16.0, 22.0, 60.0], device="cuda")
    more = dict(groups=ints([0, 2]), prefix_lens=ints([length])) if shared else {}
    o, lse = basp.attn_decode_shared(q, k, v, table, ints([length] * b), scale=0.1, slopes=slopes,
                                     **more)
    at = (length - 1) // page, slice(None), (length - 1) % page
    K, V = (x[at].repeat_interleave(2, 0) for x in (k, v))
    assert torch.equal(o, V.expand(b, -1, -1))
    want = (q.double() * K.double()).sum(-1) * 0.1
    mag = (q.double() * K.double()).abs().sum(-1) * 0.1
    check("lse", lse, want, (d + 16) * U32 * mag + 2.0 ** -18, F32)
