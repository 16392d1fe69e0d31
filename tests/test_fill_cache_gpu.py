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


@pytest.mark.parametrize("in_place", [True, False])
def test_captured_prompt(in_place):
    """A forward and the cache's filling in one graph, replayed on new shards, against eager ones."""
    b, S, H, H_kv, d, G, rank, page = 2, 512, 8, 4, 128, 2, 1, 64
    w = small_workload(b=b, S=S, H=H, H_kv=H_kv, d=d, G=G, rank=rank, seed=23)
    dev = lambda x: [s.cuda() for s in shards_of(x, w)]  # noqa: E731
    sh = RankShare(*(dev(t) for t in global_tensors(w)), G=G, rank=rank, scale=w.scale)
    mp = S // page
    table = torch.randperm(b * mp, generator=torch.Generator().manual_seed(2)).view(b, mp).to(I32).cuda()
    one, two = (PagedKV(b * mp, sh.Hkl, d, page=page) for _ in range(2))

    def prompt(cache):
        (sh.forward_sharded if in_place else sh.forward)()
        sh.fill_cache(cache, table)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        prompt(one)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            prompt(one)
    g = torch.Generator("cuda").manual_seed(9)
    for i in range(4):
        for t in (*sh.q_shards, *sh.k_shards, *sh.v_shards):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        prompt(two)
        torch.cuda.synchronize()
        assert torch.equal(one.k_pages, two.k_pages) and torch.equal(one.v_pages, two.v_pages), i
        k, _ = two.read(table, S)
        h = rank * H_kv // G
        assert torch.equal(k, torch.cat(sh.k_shards, 1)[:, :, h:h + sh.Hkl]), i
