"""Attention of one token where scores or sums leave fp32's range, in one unit of keys, over several and
over many workgroups."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
LENGTHS = [1, 5, 128, 300, 5000]


def _cache(n, n_k, d, page=64):
    mp = -(-n // page)
    g = torch.Generator("cuda").manual_seed(n)
    kp, vp = (torch.randn(mp, n_k, page, d, generator=g, device="cuda").to(BF16) for _ in range(2))
    table = torch.randperm(mp, generator=torch.Generator().manual_seed(n)).view(1, mp).to(I32).cuda()
    return kp, vp, table, torch.tensor([n], dtype=I32, device="cuda")


def _query(n_q, d):
    return (torch.rand(1, n_q, d, generator=torch.Generator("cuda").manual_seed(1), device="cuda") + 0.5).to(BF16)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("n", LENGTHS)
def test_no_key_left(n, d):
    """All scores of one kv head minus infinity: NaN and -inf there, the other head as it is."""
    kp, vp, table, lens = _cache(n, 2, d)
    q = _query(6, d)
    want = basp.attn_decode(q, kp, vp, table, lens)
    kp[:, 1] = -math.inf
    o, lse = basp.attn_decode(q, kp, vp, table, lens)
    assert o[0, 3:].isnan().all() and (lse[0, 3:] == -math.inf).all()
    assert torch.equal(o[0, :3], want[0][0, :3]) and torch.equal(lse[0, :3], want[1][0, :3])


@pytest.mark.parametrize("n", LENGTHS)
def test_a_score_of_plus_infinity(n):
    kp, vp, table, lens = _cache(n, 1, 128)
    t = n // 2
    kp[int(table[0, t // 64]), 0, t % 64, 3] = math.inf
    o, lse = basp.attn_decode(_query(3, 128), kp, vp, table, lens)
    assert o.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", LENGTHS)
def test_values_up_to_the_range_of_the_sum(n, d):
    """Equal scores and equal values whose sum is below 2^128: their mean, exactly."""
    kp, vp, table, lens = _cache(n, 1, d)
    top = 2.0 ** (127 - math.ceil(math.log2(n + 1)))
    vp.fill_(top)
    o, lse = basp.attn_decode(torch.zeros(1, 4, d, dtype=BF16, device="cuda"), kp, vp, table, lens)
    assert (o == top).all()
    assert ((lse - math.log(n)).abs() <= 2.0 ** -22 * (1 + math.log(n))).all()
