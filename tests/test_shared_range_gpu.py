"""Capped scores at both ends of the cap in decode over shared prefixes: values of any size, and prefixes
of one key."""
import pytest
import torch

from test_shared_decode_gpu import BF16, E4M3, Case, _slopes

pytestmark = pytest.mark.gpu


def _share_again(c, sizes):
    """The page that a prefix ends in, the same in every sequence's copy."""
    first, page = 0, c.cache.k_pages.shape[2]
    for n, p in zip(sizes, c.prefix.tolist()):
        if p % page:
            at = [int(c.table[s, p // page]) for s in range(first, first + n)]
            for pool in (c.cache.k_pages, c.cache.v_pages):
                raw = pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)
                raw[at, :, :p % page] = raw[at[:1], :, :p % page]
        first += n


# prefix workgroups of 64 and of 128 rows; the plan in a workgroup and in a kernel of its own
@pytest.mark.parametrize("sizes,n_q,n_k", [([3, 2], 4, 2), ([5], 40, 1), ([2] * 150, 4, 2)])
@pytest.mark.parametrize("cap", [50.0, 64.0, 200.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("power", [64, -64])
def test_values_of_any_size(sizes, n_q, n_k, cap, bias, dtype, power):
    """Scores of 3 to 5 caps (a scale of 0.1), of one sign in a sequence: minus in every third; values of
    some 2^power."""
    b, d = sum(sizes), 128
    own = [(10, 0, 40, 1, 129)[s % 5] for s in range(b)]
    c = Case(sizes, [300 - g % 7 for g in range(len(sizes))], own, n_q, n_k, d, 32, dtype, seed=b)
    g = torch.Generator("cuda").manual_seed(b)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    sign = torch.where(torch.arange(b, device="cuda") % 3 == 0, -1.0, 1.0).view(b, 1, 1)
    c.q = (sign * (1 + 0.1 * rn(b, n_q, d)) * (cap / 64)).to(BF16)
    c.cache.k_pages.copy_((1 + 0.1 * rn(*c.cache.k_pages.shape)) * (1 if dtype == E4M3 else 20))
    v = rn(*c.cache.v_pages.shape)
    if dtype == E4M3:
        c.cache.k_scales.fill_(127 + 4)
        c.cache.v_scales.fill_(127 + power)
    else:
        v = v * 2.0 ** power
    c.cache.v_pages.copy_(v)
    _share_again(c, sizes)
    c.check(cap=cap, slopes=_slopes(n_q) if bias else None)


@pytest.mark.parametrize("cap", [None, 30.0, 64.0, 100.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_prefixes_of_one_key(cap, bias, d):
    """O of a sequence whose only key is its group's prefix is that key's V, bit for bit, whatever the
    score: only its weight is formed, and divided by itself."""
    c = Case([5, 3], [1, 1], [0] * 8, 8, 2, d, 16, BF16, seed=3)
    o, _ = c.run(cap, _slopes(8) if bias else None)
    for s in range(8):
        v = c.cache.v_pages[c.table[s, 0], :, 0]
        assert torch.equal(o[s], v.repeat_interleave(4, 0))
