"""Gradients of attention over spans on sequences of millions of tokens, where a unit of the key pass sees
thousands of steps of rows."""
import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import U16, U32, check

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.mark.parametrize("S,n_q,d", [((1 << 22) + 5, 2, 64), (2300001, 1, 128)])
def test_all_rows_see_the_same_keys(S, n_q, d):
    """Every row sees keys 3 .. 40 only: one key tile with every step of every chunk of rows on its
    list, the others with none.  dK and dV against fp64 sums over all rows."""
    g = torch.Generator("cuda").manual_seed(S)
    rn = lambda n: torch.randn(1, S, n, d, generator=g, device="cuda", dtype=BF16)  # noqa: E731
    q, k, v, do = rn(n_q), rn(1), rn(1), rn(n_q)
    spans = torch.tensor([3, 40], dtype=torch.int32, device="cuda").expand(1, S, 2).contiguous()
    scale = d ** -0.5
    print(f"case {S} {n_q} {d}", flush=True)
    o, lse = basp.attn_span_fwd(q, k, v, spans, scale=scale)
    dq, dk, dv = basp.attn_span_bwd(q, k, v, o, lse, do, spans, scale=scale)
    torch.cuda.synchronize()
    K, V = k[0, 3:40, 0].double(), v[0, 3:40, 0].double()
    n = K.shape[0]
    rk, rv, ek, ev = (torch.zeros(n, d, dtype=F64, device="cuda") for _ in range(4))
    for i0 in range(0, S, 1 << 19):
        at = slice(i0, min(S, i0 + (1 << 19)))
        for h in range(n_q):
            Q, dO, O = (x[0, at, h].double() for x in (q, do, o))
            s = torch.mm(Q, K.t().contiguous()) * scale
            e = torch.mm(Q.abs(), K.abs().t().contiguous()) * scale * (d + 8) * U32
            L = lse[0, h, at].double()[:, None]
            p = torch.exp(s - L)
            ep = p * (U16 + 2.0 ** -20 + e + 14 * U32 * (s.abs() + L.abs()))
            x = torch.mm(dO, V.t().contiguous()) - (dO * O).sum(1, keepdim=True)
            ex = (d + 8) * U32 * (torch.mm(dO.abs(), V.abs().t().contiguous())
                                  + (dO * O).abs().sum(1, keepdim=True))
            ds, eds = p * x, ep * x.abs() + p * (ex + 4 * U32 * x.abs())
            rv += torch.mm(p.t().contiguous(), dO)
            rk += torch.mm(ds.t().contiguous(), Q) * scale
            # fp32 sums of all rows: 64 at a time in a chunk, 16 chunks and two halves
            ev += torch.mm((ep + (S / 16 + 64) * U32 * p).t().contiguous(), dO.abs())
            ek += torch.mm((eds + (S / 16 + 64) * U32 * ds.abs()).t().contiguous(), Q.abs()) * scale
            if i0 == 0 or at.stop == S:
                want = torch.mm(ds, K) * scale
                bound = torch.mm(eds + 64 * U32 * ds.abs(), K.abs()) * scale * 1.02
                check(f"dq {h}", dq[0, at, h], want, bound + 2.0 ** -126, F32)
    check("dk", dk[0, 3:40, 0], rk, ek * 1.02, F32)
    check("dv", dv[0, 3:40, 0], rv, ev * 1.02, F32)
    for x in (dk, dv):
        assert (x[0, :3] == 0).all() and (x[0, 40:] == 0).all()
