"""Capped scores at both ends of the cap with very large and very small values: the exponents' reference
of caps up to 64 stands still, so weights reach 2^92 and fall to 2^-92, and the products with V must stay
in fp32's range all the same."""
import pytest
import torch

import paper_2609_03151_amd as basp
import span_ref
from ops_ref import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _saturated(b, S, n_q, n_k, d, scale, cap, seed):
    """Q and K whose scores are some 3 to 5 caps, of one sign in a row: minus in every third."""
    g = torch.Generator("cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    sign = torch.where(torch.arange(S, device="cuda") % 3 == 0, -1.0, 1.0).view(1, S, 1, 1)
    q = sign * (1 + 0.1 * rn(b, S, n_q, d))
    k = (1 + 0.1 * rn(b, S, n_k, d)) * (4 * cap / (scale * d))
    return q.to(BF16), k.to(BF16), rn(b, S, n_k, d)


# 64 rows a workgroup, 128 of eight waves, 128 of four (by length, by rows)
@pytest.mark.parametrize("b,S,n_q,n_k", [(1, 1, 2, 1), (2, 300, 4, 2), (1, 900, 40, 4), (2, 500, 32, 8),
                                         (1, 1200, 64, 8)])
@pytest.mark.parametrize("cap", [50.0, 64.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("size", [2.0 ** 64, 2.0 ** -64])
def test_values_of_any_size(b, S, n_q, n_k, cap, bias, size):
    d = 64 if n_q == 40 else 128
    q, k, v = _saturated(b, S, n_q, n_k, d, 0.1, cap, S)
    v = (v * size).to(BF16)
    slopes = 2.0 ** -torch.arange(1, n_q + 1, dtype=F32, device="cuda") if bias else None
    gen = torch.Generator().manual_seed(S)
    docs, pre = span_ref.documents(b, S, max(1, S // 2), S // 4, 0, gen)
    spans = basp.attn_spans(docs.cuda(), pre.cuda())
    print(f"case {b} {S} {n_q} {cap} {bias} {size}", flush=True)
    o, lse = basp.attn_span_fwd(q, k, v, spans, scale=0.1, cap=cap, slopes=slopes)
    O, bound, L, bl = span_ref.fwd_ref(q, k, v, spans, 0.1, cap, slopes)
    check("o", o, O, bound, BF16)
    check("lse", lse, L, bl, F32)


@pytest.mark.parametrize("n_q", [4, 60])
def test_one_large_value(n_q):
    """One value of 2^100 in a row whose scores are at the cap, the others of size 1."""
    S, d, cap = 800, 128, 64.0
    q, k, v = _saturated(1, S, n_q, 2, d, 0.1, cap, 7)
    v = v.to(BF16)
    v[0, 77, 1, 9] = 2.0 ** 100
    o, lse = basp.attn_span_fwd(q, k, v, None, scale=0.1, cap=cap)
    O, bound, L, bl = span_ref.fwd_ref(q, k, v, None, 0.1, cap, None)
    check("o", o, O, bound, BF16)
    check("lse", lse, L, bl, F32)
