"""Rows of few keys: what rounds and what does not."""
import pytest
import torch

import paper_2609_03151_amd as basp

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("b,S,n", [(1, 70, 2), (2, 3000, 4), (4, 4096, 4), (6, 4100, 4)])
@pytest.mark.parametrize("cap", [None, 30.0, 100.0])
@pytest.mark.parametrize("bias", [False, True])
def test_rows_of_one_key(b, S, n, cap, bias):
    """O of a row that sees one key is that key's V, bit for bit, whatever the score: only its P is
    formed, and divided by itself (the quotient off by some 2^-23, V by 2^-9 and more apart)."""
    g = torch.Generator("cuda").manual_seed(S)
    rn = lambda n: torch.randn(b, S, n, 128, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, k, v = 2 * rn(n), rn(n), rn(n)
    at = torch.randint(0, S, (b, S), generator=g, device="cuda")
    spans = torch.stack((at, at + 1), -1).to(torch.int32)
    slopes = 2.0 ** -torch.arange(1, n + 1, dtype=F32, device="cuda") if bias else None
    o, lse = basp.attn_span_fwd(q, k, v, spans, cap=cap, slopes=slopes)
    want = torch.stack([v[i, at[i]] for i in range(b)])
    assert torch.equal(o, want)
