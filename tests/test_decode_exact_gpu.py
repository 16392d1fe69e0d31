"""Attention of one token over the cache against fp64, within the errors of weights of two bf16 and fp32
sums: short sequences, where a weight's rounding shows, values that tell every run of keys from
the others, and batches with more heads than workgroups."""
import pytest
import torch

import paper_2609_03151_amd as basp
from decode_bound import decode_exact, unit_values
from ops_ref import check, quantise_ref

pytestmark = pytest.mark.gpu
BF16, F32, E4M3, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32


def _run(q, k, v, lens, page, e4m3, max_len=None, empty=()):
    """attn_decode over a cache filled with k, v, in a workspace of the reported size inside a larger
    buffer, all bits of which are set; slots listed in `empty` have no sequence."""
    b, n_q, d = q.shape
    T, n_k = k.shape[1:3]
    lens = [0 if s in empty else n for s, n in enumerate(lens)]
    mp = -(-T // page)
    fill = torch.full((2, b * mp, n_k, page, d), 0x7F if e4m3 else -1,
                      dtype=torch.uint8 if e4m3 else torch.int16, device="cuda")
    kp, vp = fill.view(E4M3 if e4m3 else BF16)
    kw = {}
    if e4m3:
        kw = {n: torch.full((b * mp, n_k, page), 255, dtype=torch.uint8, device="cuda")
              for n in ("k_scales", "v_scales")}
    table = torch.randperm(b * mp, generator=torch.Generator().manual_seed(T)).view(b, mp).to(I32).cuda()
    ints = torch.tensor(lens, dtype=I32, device="cuda")
    print("decode", tuple(q.shape), tuple(k.shape), e4m3, lens[:6], len(empty), flush=True)
    basp.kv_write(k, v, kp, vp, table, torch.zeros_like(ints), count=ints, **kw)
    max_len = T if max_len is None else max_len
    need = basp.attn_decode_workspace_bytes(b, n_q, n_k, d, max_len)
    buf = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    ws = buf[256:256 + need]
    o, lse = basp.attn_decode(q, kp, vp, table, ints, max_len=max_len, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert (buf[:256] == 255).all() and (buf[256 + need:] == 255).all()
    K, V = (quantise_ref(x)[0] for x in (k, v)) if e4m3 else (k, v)
    ro, bo, rl, bl = decode_exact(q, K, V, lens, d ** -0.5, max_len)
    check("o", o, ro, bo, BF16)
    check("lse", lse, rl, bl, F32)
    again = basp.attn_decode(q, kp, vp, table, ints, max_len=max_len, **kw)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def _randn(*s, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*s, generator=g, device="cuda")


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_q,n_k", [(8, 2), (5, 1), (20, 1), (70, 2)])
def test_weights_keep_two_bf16(d, e4m3, n_q, n_k):
    """Up to 48 keys: what a weight of one bf16 is off by is several times the bound."""
    lens = list(range(49))
    q = (_randn(49, n_q, d, seed=d) * 1.5).to(BF16)
    k, v = (_randn(49, 48, n_k, d, seed=s).to(BF16) for s in (1, 2))
    _run(q, k, v, lens, 16, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("b,L,n_q,n_k,d,page", [
    (1, 70001, 8, 1, 128, 64), (1, 33333, 4, 4, 64, 16), (2, 20000, 32, 8, 96, 256),
    (6, 9001, 7, 1, 80, 32), (64, 3000, 8, 2, 128, 64), (3, 6000, 40, 2, 128, 128),
    (2, 50000, 33, 1, 64, 64)])
def test_every_unit_in_its_place(e4m3, b, L, n_q, n_k, d, page):
    """One head over all workgroups to many heads a workgroup."""
    g = torch.Generator().manual_seed(L)
    lens = [L] + torch.randint(0, L + 1, (b - 1,), generator=g).tolist()
    q = (_randn(b, n_q, d, seed=3) * 0.5).to(BF16)
    _run(q, _randn(b, L, n_k, d, seed=4).to(BF16), unit_values(b, L, n_k, d, "cuda"), lens, page, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("b,n_q,n_k,L,d", [(800, 2, 1, 300, 64), (130, 16, 8, 700, 128),
                                           (600, 20, 1, 260, 80), (300, 40, 2, 500, 96),
                                           (768, 1, 1, 200, 128), (1600, 3, 1, 140, 64)])
@pytest.mark.parametrize("share_empty", [0.0, 0.5, 0.97, 1.0])
def test_more_heads_than_workgroups(e4m3, b, n_q, n_k, L, d, share_empty):
    """A workgroup's run crosses heads and sequences, empty ones between them, and its last head alone can
    go on in the next; where most are empty there are fewer units than workgroups."""
    g = torch.Generator().manual_seed(b)
    lens = torch.randint(1, L + 1, (b,), generator=g).tolist()
    lens[b // 2] = L
    gone = (torch.rand(b, generator=g) < share_empty).tolist()
    gone[b // 2] = share_empty == 1.0
    q = (_randn(b, n_q, d, seed=3) * 0.5).to(BF16)
    _run(q, _randn(b, L, n_k, d, seed=4).to(BF16), unit_values(b, L, n_k, d, "cuda"), lens, 32, e4m3,
         empty={s for s in range(b) if gone[s]})


@pytest.mark.parametrize("max_len", [129, 1000, 5000])
def test_a_longer_max_len_changes_the_cut_alone(max_len):
    """Few keys of many allowed: idle workgroups, and descriptors by head."""
    b, n_q, n_k, d, L = 5, 8, 2, 128, 129
    q = _randn(b, n_q, d, seed=3).to(BF16)
    k, v = (_randn(b, L, n_k, d, seed=s).to(BF16) for s in (1, 2))
    _run(q, k, v, [129, 0, 1, 128, 64], 64, False, max_len=max_len)
