"""Infinities and NaN that nobody sees in the backward's wider workgroups (128 and 256 query rows of the dQ
pass): gradients of the other rows to their bounds, zeros where nothing is seen."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp
import span_ref
from ops_ref import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(b, S, n_q, n_k, d, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    rn = lambda n: torch.randn(b, S, n, d, generator=g, device="cuda").to(BF16)  # noqa: E731
    return 2 * rn(n_q), rn(n_k), rn(n_k), rn(n_q)


# 25K and 65K query rows: 128 a workgroup; 108K: 256
@pytest.mark.parametrize("n_q,n_k", [(14, 2), (36, 4), (60, 4)])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("cap", [None, 30.0, 100.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_garbage_documents(n_q, n_k, d, cap, bias, bad):
    b, S = 2, 900
    q, k, v, do = _inputs(b, S, n_q, n_k, d, seed=d + n_q)
    docs = torch.zeros(b, S, dtype=torch.int32)
    docs[:, 300:] = 1            # garbage
    docs[:, 411:] = 2
    docs[1, 850:] = -1           # padding
    spans = basp.attn_spans(docs.cuda(), torch.full((b, S), 100).cuda())
    live = torch.ones(b, S, dtype=torch.bool, device="cuda")
    live[:, 300:411] = False
    live[1, 850:] = False
    slopes = 2.0 ** -torch.arange(1, n_q + 1, dtype=F32, device="cuda") if bias else None
    rule = dict(scale=0.1, cap=cap, slopes=slopes)
    o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
    q2, k2, v2, do2 = (torch.where(live[..., None, None], x, bad) for x in (q, k, v, do))
    o2, lse2 = basp.attn_span_fwd(q2, k2, v2, spans, **rule)
    print(f"case {n_q} {d} {cap} {bias} {bad}", flush=True)
    got = basp.attn_span_bwd(q2, k2, v2, o2, lse2, do2, spans, grad_dtype=BF16, **rule)
    o = torch.where(live[..., None, None], o2, o)
    lse = torch.where(live[:, None], lse2, lse)
    ref = span_ref.bwd_ref(q, k, v, o, lse, do, spans, *rule.values())
    for name, x, (r, bound) in zip(("dq", "dk", "dv"), got, ref):
        check(name, x[live], r[live], bound[live], BF16)
        assert (x[1, 850:] == 0).all(), name
        assert not x[:, 300:411].isfinite().any(), name


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("cap", [None, 30.0])
def test_causal(d, cap):
    """43K query rows, causal: 256 a workgroup.  A last key or value of no finite number reaches the
    last row alone, and through its weights and products dK and dV."""
    b, S, n_q, n_k = 2, 901, 24, 4
    q, k, v, do = _inputs(b, S, n_q, n_k, d, seed=d)
    o, lse = basp.attn_span_fwd(q, k, v, None, scale=0.1, cap=cap)
    ref = span_ref.bwd_ref(q, k, v, o, lse, do, None, 0.1, cap, None)
    for name, bad in (("v", math.inf), ("v", math.nan), ("k", math.nan)):
        x = {"k": k.clone(), "v": v.clone()}
        x[name][:, -1] = bad
        print(f"case {d} {cap} {name} {bad}", flush=True)
        o2, lse2 = basp.attn_span_fwd(q, x["k"], x["v"], None, scale=0.1, cap=cap)
        assert not o2[:, -1].isfinite().any()
        # what the rows before the last get, from the clean forward's outputs there
        oc, lc = o.clone(), lse.clone()
        oc[:, -1], lc[..., -1] = o2[:, -1], lse2[..., -1]
        dq, dk, dv = basp.attn_span_bwd(q, x["k"], x["v"], oc, lc, do, None, scale=0.1, cap=cap,
                                        grad_dtype=BF16)
        r, bound = ref[0]
        check("dq", dq[:, :-1], r[:, :-1], bound[:, :-1], BF16)
        assert not dq[:, -1].isfinite().any() and not dk.isfinite().any()
        if name == "v":          # the weights stay
            check("dv", dv, *ref[2], BF16)
        else:
            assert not dv.isfinite().any()
