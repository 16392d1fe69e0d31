"""The bound that attention of one token is held to, on the CPU: the steps that the kernel documents
stay inside it, and mistakes planted in them do not."""
import math

import pytest
import torch

from decode_bound import UNIT, decode_exact, unit_values
from ops_ref import F64, check

BF16, F32 = torch.bfloat16, torch.float32


def _inputs(b, T, n_q, n_k, d, q_size, seed=3):
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return ((rn(b, n_q, d) * q_size).to(BF16), rn(b, T, n_k, d).to(BF16), rn(b, T, n_k, d).to(BF16))


def _steps(q, k, v, lens, scale, parts=2, lost=None, swapped=None):
    """O as the kernel forms it, in bf16: fp32 scores, weights as the sum of `parts` bf16, units of keys
    added one after the other; `lost`: a unit whose products are left out, `swapped`: two units of
    which the second's are taken for both (their weights stay)."""
    b, n_q, d = q.shape
    n_k = k.shape[2]
    out = []
    for s, n in enumerate(lens):
        if n == 0:
            out.append(torch.zeros(n_q, d))
            continue
        K, V = k[s, :n].float().transpose(0, 1), v[s, :n].float().transpose(0, 1)
        S = torch.matmul(q[s].float().view(n_k, -1, d), K.transpose(1, 2).contiguous()) * scale
        w = torch.exp(S - S.amax(-1, keepdim=True))
        hi = w.to(BF16).float()
        W = hi + (w - hi).to(BF16).float() if parts == 2 else hi
        prod = [torch.matmul(W[..., i:i + UNIT], V[:, i:i + UNIT]) for i in range(0, n, UNIT)]
        if lost is not None:
            prod[lost] = torch.zeros_like(prod[0])
        if swapped is not None:
            prod[swapped[0]] = prod[swapped[1]]
        out.append((sum(prod) / w.sum(-1, keepdim=True)).view(n_q, d))
    return torch.stack(out).to(BF16)


@pytest.mark.parametrize("n_q,n_k,d", [(8, 2, 128), (4, 1, 64), (6, 2, 96)])
def test_a_weight_of_one_bf16_is_outside(n_q, n_k, d):
    lens = list(range(49))
    q, k, v = _inputs(len(lens), 48, n_q, n_k, d, 1.5)
    ref, bound, _, _ = decode_exact(q, k, v, lens, d ** -0.5)
    check("two", _steps(q, k, v, lens, d ** -0.5), ref, bound, BF16)
    with pytest.raises(AssertionError):
        check("one", _steps(q, k, v, lens, d ** -0.5, parts=1), ref, bound, BF16)


@pytest.mark.parametrize("T,n_q,n_k,d", [(70001, 2, 1, 128), (20000, 4, 2, 64), (700, 2, 1, 80)])
def test_a_unit_in_the_wrong_place_is_outside(T, n_q, n_k, d):
    q, k, _ = _inputs(1, T, n_q, n_k, d, 0.5)
    v = unit_values(1, T, n_k, d, "cpu")
    ref, bound, _, _ = decode_exact(q, k, v, [T], d ** -0.5)
    check("right", _steps(q, k, v, [T], d ** -0.5), ref, bound, BF16)
    last = (T - 1) // UNIT
    for wrong in (dict(lost=0), dict(lost=last // 2), dict(lost=last), dict(swapped=(1, 0)),
                  dict(swapped=(last // 2, last)), dict(swapped=(0, min(d, last - 1)))):
        with pytest.raises(AssertionError):
            check(str(wrong), _steps(q, k, v, [T], d ** -0.5, **wrong), ref, bound, BF16)


def test_bound_of_the_sum():
    """LSE in fp32, and of a sequence without keys."""
    q, k, v = _inputs(3, 500, 4, 1, 64, 1.5)
    lens = [500, 0, 1]
    _, _, ref, bound = decode_exact(q, k, v, lens, 0.125)
    s = torch.matmul(q.float(), k[:, :, 0].float().transpose(1, 2).contiguous()) * 0.125
    got = torch.stack([torch.logsumexp(s[i, :, :n], -1) if n else torch.full((4,), -math.inf)
                       for i, n in enumerate(lens)])
    check("lse", got, ref, bound, F32)
    with pytest.raises(AssertionError):   # one key of 500 left out
        check("lse", torch.logsumexp(s[:1, :, 1:], -1), ref[:1], bound[:1], F32)
    assert ref.dtype == F64
