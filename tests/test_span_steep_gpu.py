"""Slopes so steep that every row sees its own key alone."""
import pytest
import torch

import paper_2609_03151_amd as basp
import span_ref
from ops_ref import TINY, U16, U32, check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


# 64 and 128 rows a workgroup of the forward, 64, 128 and 256 of the backward
@pytest.mark.parametrize("b,S,n_q,n_k", [(2, 333, 4, 2), (1, 1100, 40, 4), (2, 1500, 40, 4)])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("cap", [None, 30.0, 100.0])
@pytest.mark.parametrize("kind", ["causal", "docs", "all"])
@pytest.mark.parametrize("power", [12, 18, 30, 60])
def test_steep_slopes(b, S, n_q, n_k, d, cap, kind, power):
    """O is the row's V, bit for bit where the reference of its weight is its own score (no cap, or one
    past 64), else to its weight's one rounding; the LSE is its own score; dV the sum of dO over the heads, and dS what
    rounding leaves of dO.V - dO.O = 0."""
    g = torch.Generator("cuda").manual_seed(S + d)
    rn = lambda n: torch.randn(b, S, n, d, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, k, v, do = rn(n_q), rn(n_k), rn(n_k), rn(n_q)
    slopes = 2.0 ** power * torch.linspace(1, 2, n_q, device="cuda")
    if kind == "causal":
        spans = None
    elif kind == "all":
        spans = torch.tensor([0, S], dtype=torch.int32).expand(b, S, 2).contiguous().cuda()
    else:
        docs, pre = span_ref.documents(b, S, S // 4, S // 9, 0, torch.Generator().manual_seed(S))
        spans = basp.attn_spans(docs.cuda(), pre.cuda())
    print(f"case {b} {S} {n_q} {d} {cap} {kind} {power}", flush=True)
    o, lse = basp.attn_span_fwd(q, k, v, spans, scale=0.1, cap=cap, slopes=slopes)
    rep = n_q // n_k
    K, V = (x.double().repeat_interleave(rep, 2) for x in (k, v))
    if cap == 30.0:
        check("o", o, V, (U16 + 2.0 ** -20) * V.abs(), BF16)
    else:
        assert torch.equal(o.double(), V)
    Q, dO = q.double(), do.double()
    s, mag = (Q * K).sum(-1) * 0.1, (Q * K).abs().sum(-1) * 0.1
    e = (d + 16) * U32 * mag + 2.0 ** -18
    if cap:
        s, e = cap * torch.tanh(s / cap), e + cap * 2.0 ** -20
    check("lse", lse, s.transpose(1, 2), e.transpose(1, 2), F32)
    dq, dk, dv = basp.attn_span_bwd(q, k, v, o, lse, do, spans, scale=0.1, cap=cap, slopes=slopes)
    group = lambda x: x.view(b, S, n_k, rep, d).sum(3)  # noqa: E731
    # P is 1 but for the exponent's error, then a bf16 number; dO.V and dO.O of d terms
    ep = U16 + 4 * e[..., None] + 2.0 ** -17
    ds = (2 * d + 16) * U32 * (dO * V).abs().sum(-1, keepdim=True) * 1.1
    if cap == 30.0:  # O is off V by its weight's rounding and its own
        ds = ds + 2.02 * U16 * (dO * V).abs().sum(-1, keepdim=True)
    check("dv", dv, group(dO), group(ep * dO.abs()) + TINY, F32)
    check("dq", dq, torch.zeros_like(Q), 0.1 * ds * K.abs() * 1.1 + TINY, F32)
    check("dk", dk, torch.zeros_like(group(Q)), 0.1 * group(ds * Q.abs()) * 1.1 + TINY, F32)
