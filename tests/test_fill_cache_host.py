"""Which K and V a share puts into a cache: those of its last forward, packed or in place (the kernels
replaced by plain indexing, on the CPU)."""
import pytest
import torch

from paper_2609_03151_amd import share

G, b, Sg, d = 4, 2, 6, 64
S = G * Sg


class Cache:
    """Rows [b, S, n_kv, d] in the place of pages."""

    def __init__(self, n_kv):
        self.k, self.v = (torch.full((b, S, n_kv, d), torch.nan) for _ in range(2))

    def write(self, k, v, block_table, start):
        assert start.dtype == torch.int32 and start.shape == (b,) and start.is_contiguous()
        for s in range(b):
            at = slice(int(start[s]), int(start[s]) + k.shape[1])
            assert self.k[s, at].isnan().all()   # every token once
            self.k[s, at], self.v[s, at] = k[s].float(), v[s].float()


def _share(monkeypatch, H_kv, rank, norm_rope=None):
    """(the share, K and V of its heads over the whole sequence)."""
    g = torch.Generator().manual_seed(H_kv)
    new = lambda n: [torch.randn(b, Sg, n, d, generator=g).to(torch.bfloat16) for _ in range(G)]  # noqa: E731
    h = rank * H_kv // G

    def packed(shards, n):
        return torch.cat(shards, 1)[:, :, h:h + n]

    def pack_qkv(q_shards, k_shards, v_shards, r, q, k, v):
        k.copy_(packed(k_shards, k.shape[2])), v.copy_(packed(v_shards, v.shape[2]))

    def norm(q, k, *a, q_out, k_out, **kw):
        k_out.copy_(-2 * k)

    for name, f in (("pack_qkv", pack_qkv), ("qk_norm_rope", norm)):
        monkeypatch.setattr(share, name, f)
    for name in ("attn_fwd", "unpack", "attn_fwd_sharded"):
        monkeypatch.setattr(share, name, lambda *a, **k: None)
    sh = share.RankShare(new(8), new(H_kv), new(H_kv), None, G=G, rank=rank, norm_rope=norm_rope)
    for t in (sh.k, sh.v):
        t.fill_(7.0)   # what the constructor leaves there is anything

    def replace():
        """The next prompt's shards, in place."""
        for t in (*sh.k_shards, *sh.v_shards):
            t.copy_(torch.randn(t.shape, generator=g))

    return sh, lambda: (packed(sh.k_shards, sh.Hkl).float(), packed(sh.v_shards, sh.Hkl).float()), replace


def _filled(sh):
    c = Cache(sh.Hkl)
    sh.fill_cache(c, None)
    return c.k, c.v


@pytest.mark.parametrize("H_kv,rank", [(8, 3), (4, 1), (2, 0), (2, 3), (1, 2)])
def test_the_last_forward_fills_the_cache(monkeypatch, H_kv, rank):
    sh, want, replace = _share(monkeypatch, H_kv, rank)
    sh.forward_sharded()
    assert all(torch.equal(x, y) for x, y in zip(_filled(sh), want()))
    replace()
    sh.forward()
    first = want()
    replace()          # the next prompt has come in; the last forward's K and V are the packed ones
    assert all(torch.equal(x, y) for x, y in zip(_filled(sh), first))
    sh.forward_sharded()
    assert all(torch.equal(x, y) for x, y in zip(_filled(sh), want()))
    assert torch.equal(sh.k.float(), first[0])   # which a backward of the first may need
    sh.pack_qkv()      # the steps one by one
    assert all(torch.equal(x, y) for x, y in zip(_filled(sh), want()))


def test_no_forward_no_cache(monkeypatch):
    sh, _, _ = _share(monkeypatch, 4, 1)
    with pytest.raises(RuntimeError, match="forward"):
        _filled(sh)


def test_with_norm_the_keys_are_the_rotated_ones(monkeypatch):
    none = share.QkNormRope(None, None, None, None)
    sh, want, _ = _share(monkeypatch, 4, 2, none)
    sh.pack_qkv()      # V is the new prompt's, K not yet
    with pytest.raises(RuntimeError, match="forward"):
        _filled(sh)
    with pytest.raises(ValueError):
        sh.forward_sharded()
    sh.forward()
    k, v = _filled(sh)
    assert torch.equal(k, -2 * want()[0]) and torch.equal(v, want()[1])
