"""A share with a score rule: what it refuses (host only)."""
import pytest
import torch

from paper_2609_03151_amd.share import RankShare, ScoreRule


def _shards(n):
    return [torch.zeros(1, 256, n, 64, dtype=torch.bfloat16) for _ in range(2)]


def test_refusals():
    q, k = _shards(4), _shards(2)
    with pytest.raises(ValueError):  # the slopes of a rank's own heads only
        RankShare(q, k, k, q, 2, 0, rule=ScoreRule(slopes=torch.ones(2)))
    sh = RankShare(q, k, k, q, 2, 1, rule=ScoreRule(cap=5.0, slopes=torch.arange(4.0)))
    assert sh.slopes.tolist() == [2.0, 3.0]
    with pytest.raises(ValueError):
        sh.forward_sharded()
    with pytest.raises(ValueError):
        sh.backward_sharded()
    with pytest.raises(TypeError):  # host tensors: the library has no other way to compute
        sh.attn_fwd()
