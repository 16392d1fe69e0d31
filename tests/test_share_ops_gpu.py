"""The share with norm and rotation, and generation from it: the operators in a row, as a layer uses
them, against plain fp64."""
import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import check, decode_ref, gather_ref, norm_rope_ref
from paper_2609_03151_amd.cache import PagedKV
from paper_2609_03151_amd.share import QkNormRope, RankShare
from parity import check_close
from synth_inputs import global_tensors, shards_of, small_workload

pytestmark = pytest.mark.gpu
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def _layer(d, S, seed=5):
    g = torch.Generator("cuda").manual_seed(seed)
    w = [1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    return QkNormRope(*w, *basp.rope_table(S, d, base=500000.0), eps=1e-6)


def _reference(w, n, q, k, v, do):
    """O, dQ, dK, dV, dwq, dwk of the rank's heads by fp64 autograd over the whole composition."""
    x = [t.cuda().double() for t in (q, k, v, do)]
    for t in x[:3]:
        t.requires_grad_()
    wq, wk = (t.double().requires_grad_() for t in (n.q_weight, n.k_weight))
    P = torch.arange(w.S, device="cuda")[None].expand(w.b, w.S)

    def normed(t, ww):
        y = t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + n.eps) * ww
        a, b = y.chunk(2, -1)
        c, s = n.cos.double()[P][:, :, None], n.sin.double()[P][:, :, None]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    Q, K = normed(x[0], wq), normed(x[1], wk)
    rep = Q.shape[2] // K.shape[2]
    Kr, Vr = K.repeat_interleave(rep, 2), x[2].repeat_interleave(rep, 2)
    s = torch.matmul(Q.transpose(1, 2), Kr.permute(0, 2, 3, 1).contiguous()) * w.scale
    s = s.masked_fill(torch.ones(w.S, w.S, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
    O = torch.matmul(torch.softmax(s, -1), Vr.transpose(1, 2).contiguous()).transpose(1, 2)
    return (O, *torch.autograd.grad(O, (*x[:3], wq, wk), x[3]))


@pytest.mark.parametrize("b,S,H,H_kv,d,G,rank", [(1, 384, 8, 2, 128, 2, 1), (2, 130, 8, 8, 64, 2, 0),
                                                 (1, 256, 8, 2, 96, 4, 3), (1, 320, 8, 4, 80, 1, 0)])
def test_step_with_norm_and_rotation(b, S, H, H_kv, d, G, rank):
    w = small_workload(b=b, S=S, H=H, H_kv=H_kv, d=d, G=G, rank=rank, seed=11)
    tensors = global_tensors(w)
    n = _layer(d, S)
    dev = lambda x: [s.cuda() for s in shards_of(x, w)]  # noqa: E731
    sh = RankShare(*(dev(t) for t in tensors), G=G, rank=rank, scale=w.scale, norm_rope=n)
    sh.step()
    torch.cuda.synchronize()

    def local(t, heads):
        h0, nl = w.first_head(heads), basp.heads_per_member(heads, G)
        return t[w.seq_offset:w.seq_offset + b, :, h0:h0 + nl]

    q, k, v, do = (local(t, m) for t, m in zip(tensors, (H, H_kv, H_kv, H)))
    ref = _reference(w, n, q, k, v, do)
    for name, got, r in zip(("O", "dQ", "dK", "dV"), (sh.o, sh.dq, sh.dk, sh.dv), ref):
        check_close(name, got.double().cpu().numpy(), r.detach().cpu().numpy())
    # a weight's gradient sums over b*S*heads rows the errors of theirs (each within the bar of
    # dQ, dK, and of no common sign): relative to its own size
    for name, got, r in (("dq_weight", sh.dq_weight, ref[4]), ("dk_weight", sh.dk_weight, ref[5])):
        assert (got.double() - r).norm() <= 2e-2 * r.norm(), name
    # the gradients reach the shards, and the packed Q is still what the pack gave
    assert torch.equal(sh.q_in.cpu(), q)
    Sg, h0 = S // G, w.first_head(H)
    for j in range(G):
        assert torch.equal(sh.dq_shards[j][:, :, h0:h0 + H // G], sh.dq[:, j * Sg:(j + 1) * Sg])
    with pytest.raises(ValueError):
        sh.forward_sharded()
    with pytest.raises(ValueError):
        sh.backward_sharded()


def test_share_without_norm_is_what_it_was():
    """No norm and no rotation: the same buffers and bits as the calls one by one."""
    w = small_workload(b=1, S=256, H=8, H_kv=2, d=128, G=2, rank=1, seed=3)
    dev = lambda x: [s.cuda() for s in shards_of(x, w)]  # noqa: E731
    a, c = (RankShare(*(dev(t) for t in global_tensors(w)), G=2, rank=1) for _ in range(2))
    a.step()
    assert a.q_in is a.q and a.k_in is a.k and a.dq_weight is None
    c.pack_qkv(), c.attn_fwd(), c.unpack_o(), c.pack_do(), c.attn_bwd(), c.unpack_grads()
    for n in ("q", "k", "o", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, n), getattr(c, n))


@pytest.mark.parametrize("dtype", [BF16, torch.float8_e4m3fn])
@pytest.mark.parametrize("normed", [False, True])
def test_generation_from_a_share(dtype, normed):
    """Prompt by forward(), its K and V into the cache, three tokens by decode(), one slot of the batch
    without a sequence; then the cache read back."""
    b, S, H, H_kv, d, G, rank, page, new = 2, 256, 8, 4, 128, 2, 1, 32, 3
    w = small_workload(b=b, S=S, H=H, H_kv=H_kv, d=d, G=G, rank=rank, seed=7)
    n = _layer(d, S + new) if normed else None
    dev = lambda x: [s.cuda() for s in shards_of(x, w)]  # noqa: E731
    sh = RankShare(*(dev(t) for t in global_tensors(w)), G=G, rank=rank, scale=w.scale, norm_rope=n)
    sh.forward()
    mp = -(-(S + new) // page)
    cache = PagedKV(3 * mp, sh.Hkl, d, page=page, dtype=dtype)
    table = torch.randperm(3 * mp, generator=torch.Generator().manual_seed(1)).view(3, mp).to(I32).cuda()
    sh.fill_cache(cache, table[:b].contiguous())
    g = torch.Generator("cuda").manual_seed(2)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    new_k, new_v = [], []
    for t in range(new):
        q, k, v = rn(3, 1, sh.Hl, d), rn(3, 1, sh.Hkl, d), rn(3, 1, sh.Hkl, d)
        lens = torch.tensor([S + t + 1, S + t + 1, 0], dtype=I32, device="cuda")
        o, lse = sh.decode(cache, q, k, v, table, lens)
        Q, P = q, (lens - 1).view(-1, 1)
        if normed:
            Q, kn = basp.qk_norm_rope(q, k, n.q_weight, n.k_weight, n.cos, n.sin, positions=P)
            check("k", kn, *norm_rope_ref(k, n.k_weight, n.cos, n.sin, P, n.eps, d, False), BF16)
            k = kn
        new_k.append(k[:b]), new_v.append(v[:b])
        for s in range(3):
            L = int(lens[s])
            K = gather_ref(cache.k_pages, cache.k_scales, table[s], L)
            V = gather_ref(cache.v_pages, cache.v_scales, table[s], L)
            ro, bo, rl, bl = decode_ref(Q[s, 0], K, V, w.scale)
            check("o", o[s], ro, bo, BF16)
            check("lse", lse[s], rl, bl, F32)
    # the last token's attention is the last row of attention over the whole, longer sequence
    k, v = cache.read(table[:b].contiguous(), S + new)
    want_k, want_v = torch.cat([sh.k, *new_k], 1), torch.cat([sh.v, *new_v], 1)
    if dtype == BF16:
        assert torch.equal(k, want_k) and torch.equal(v, want_v)
    else:
        for x, y in ((k, want_k), (v, want_v)):
            # half a step of e4m3 of the value, or of its least normal value at the row's scale:
            # 2^-10 of 2^e with 2^e at most the row's maximum / 224
            top = y.double().abs().amax(-1, keepdim=True)
            off = (x.double() - y.double()).abs()
            assert (off <= torch.maximum(y.double().abs() * 2.0 ** -4, top * 2.0 ** -10 / 224)).all()
