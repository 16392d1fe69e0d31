"""A share's prompt into a cache after either forward, and a token generated from it."""
import pytest
import torch

from paper_2609_03151_amd.cache import PagedKV
from paper_2609_03151_amd.share import RankShare
from synth_inputs import global_tensors, shards_of, small_workload

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("dtype", [BF16, torch.float8_e4m3fn])
@pytest.mark.parametrize("b,S,H,H_kv,d,G,rank", [(2, 512, 8, 4, 128, 2, 1), (1, 1024, 8, 2, 64, 4, 3),
                                                 (3, 1024, 8, 8, 80, 4, 2), (1, 256, 4, 4, 96, 1, 0)])
def test_either_forward_fills_the_same_cache(dtype, b, S, H, H_kv, d, G, rank):
    w = small_workload(b=b, S=S, H=H, H_kv=H_kv, d=d, G=G, rank=rank, seed=17)
    dev = lambda x: [s.cuda() for s in shards_of(x, w)]  # noqa: E731
    sh = RankShare(*(dev(t) for t in global_tensors(w)), G=G, rank=rank, scale=w.scale)
    page = 32
    mp = -(-(S + 1) // page)
    table = torch.randperm(b * mp, generator=torch.Generator().manual_seed(2)).view(b, mp).to(I32).cuda()
    g = torch.Generator("cuda").manual_seed(5)
    q, k, v = (torch.randn(b, 1, n, d, generator=g, device="cuda").to(BF16)
               for n in (sh.Hl, sh.Hkl, sh.Hkl))
    lens = torch.full((b,), S + 1, dtype=I32, device="cuda")
    got = []
    for forward in (sh.forward_sharded, sh.forward):   # in place first: nothing is packed yet
        cache = PagedKV(b * mp, sh.Hkl, d, page=page, dtype=dtype)
        forward()
        sh.fill_cache(cache, table)
        got.append((*cache.read(table, S), *sh.decode(cache, q, k, v, table, lens)))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    if dtype == BF16:
        h = rank * H_kv // G
        for x, shards in ((got[0][0], sh.k_shards), (got[0][1], sh.v_shards)):
            assert torch.equal(x, torch.cat(shards, 1)[:, :, h:h + sh.Hkl])
