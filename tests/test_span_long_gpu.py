"""Attention over spans on very long sequences, and two calls at once."""
import pytest
import torch

import paper_2609_03151_amd as basp
import span_ref
from ops_ref import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _check(inputs, outputs, size, rule, which):
    """Documents of `size` tokens against fp64 of each by itself."""
    q, k, v, do = inputs
    o, lse, *grads = outputs
    S = q.shape[1]
    rule = tuple(rule.values())
    for beta, doc in which:
        at = slice(doc * size, min(S, (doc + 1) * size))
        cut = lambda x: x[beta:beta + 1, at].contiguous()  # noqa: E731
        qs, ks, vs, dos, os = map(cut, (q, k, v, do, o))
        ls = lse[beta:beta + 1, :, at].contiguous()
        O, bo, L, bl = span_ref.fwd_ref(qs, ks, vs, None, *rule)
        check(f"o {beta} {doc}", os, O, bo, BF16)
        check(f"lse {beta} {doc}", ls, L, bl, F32)
        ref = span_ref.bwd_ref(qs, ks, vs, os, ls, dos, None, *rule)
        for name, x, (r, bound) in zip(("dq", "dk", "dv"), grads, ref):
            check(f"{name} {beta} {doc}", cut(x), r, bound, BF16)


def test_documents_of_a_long_batch():
    """Three sequences of 1.5 million tokens, tensors past 4 GiB: documents at both ends, and those
    across the bounds of the key pass's row chunks, against fp64 of each by itself."""
    b, S, n_q, n_k, d = 3, 1500007, 8, 1, 64
    assert b * S * n_q * d * 2 > 2 ** 32
    g = torch.Generator("cuda").manual_seed(1)
    rn = lambda n: torch.randn(b, S, n, d, generator=g, device="cuda", dtype=BF16)  # noqa: E731
    q, k, v, do = rn(n_q), rn(n_k), rn(n_k), rn(n_q)
    size = 701
    docs = (torch.arange(S, device="cuda") // size).expand(b, S)
    spans = basp.attn_spans(docs)
    slopes = 2.0 ** -torch.arange(1, n_q + 1, dtype=F32, device="cuda")
    rule = dict(scale=0.1, cap=20.0, slopes=slopes)
    o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
    grads = basp.attn_span_bwd(q, k, v, o, lse, do, spans, grad_dtype=BF16, **rule)
    torch.cuda.synchronize()
    last = (S - 1) // size
    _check((q, k, v, do), (o, lse, *grads), size, rule,
           ((0, 0), (0, 65536 // size), (1, 10 * 65536 // size), (2, last - 1), (2, last)))


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("cap", [None, 30.0, 100.0])
@pytest.mark.parametrize("bias", [False, True])
def test_documents_of_a_large_batch(d, cap, bias):
    """104K query rows, where the workgroups are the largest."""
    b, S, n_q, n_k, size = 2, 6503, 8, 2, 411
    g = torch.Generator("cuda").manual_seed(d)
    rn = lambda n: torch.randn(b, S, n, d, generator=g, device="cuda", dtype=BF16)  # noqa: E731
    q, k, v, do = rn(n_q), rn(n_k), rn(n_k), rn(n_q)
    spans = basp.attn_spans((torch.arange(S, device="cuda") // size).expand(b, S))
    slopes = 2.0 ** -torch.arange(1, n_q + 1, dtype=F32, device="cuda") if bias else None
    rule = dict(scale=0.1, cap=cap, slopes=slopes)
    o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
    grads = basp.attn_span_bwd(q, k, v, o, lse, do, spans, grad_dtype=BF16, **rule)
    _check((q, k, v, do), (o, lse, *grads), size, rule, [(1, i) for i in (0, 4, 5, 9, 14, 15)])


def test_two_calls_at_once():
    """Steps on two streams side by side, a workspace each: the bits of one after the other."""
    def one(seed):
        g = torch.Generator("cuda").manual_seed(seed)
        rn = lambda n: torch.randn(2, 3000, n, 128, generator=g, device="cuda").to(BF16)  # noqa: E731
        q, k, v, do = rn(4), rn(2), rn(2), rn(4)
        docs = torch.randint(0, 2, (2, 3000), generator=g, device="cuda").cumsum(1) // 200
        spans = basp.attn_spans(docs)
        ws = torch.empty(basp.attn_span_bwd_workspace_bytes(2, 3000, 4, 2, 128), device="cuda",
                         dtype=torch.uint8)
        return q, k, v, do, spans, ws

    def go(x):
        q, k, v, do, spans, ws = x
        o, lse = basp.attn_span_fwd(q, k, v, spans, cap=40.0)
        return o, lse, *basp.attn_span_bwd(q, k, v, o, lse, do, spans, cap=40.0, workspace=ws)

    inputs = [one(1), one(2)]
    want = [[t.clone() for t in go(x)] for x in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = go(inputs[i])
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(a, c) for a, c in zip(x, y))
