"""Norm and rotation of calls that move more than the last-level cache holds, which read with the
non-temporal hint: kernels of their own, for every type, head dim and pair order."""
import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import check, norm_rope_bwd_ref, norm_rope_ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HINT = 192 << 20   # bytes of a call from which on its inputs are read with the hint


def _inputs(d, dtype, bytes_per_element, b, n_q, n_k):
    """Just past the switch, with a ragged end."""
    S = HINT // (b * (n_q + n_k) * d * bytes_per_element) + 3
    assert b * S * (n_q + n_k) * d * bytes_per_element > HINT
    g = torch.Generator("cuda").manual_seed(d)
    rn = lambda *s, t=dtype: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    P = torch.arange(S, device="cuda")[None].expand(b, S)
    return rn(b, S, n_q, d), rn(b, S, n_k, d), 1 + 0.2 * rn(d, t=F32), 1 + 0.2 * rn(d, t=F32), P, rn


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward(dtype, d, inter):
    q, k, qw, kw, P, _ = _inputs(d, dtype, 2 * dtype.itemsize, 2, 7, 2)
    cos, sin = basp.rope_table(q.shape[1], d // 2)
    print("forward", tuple(q.shape), dtype, inter, flush=True)
    qo, ko = basp.qk_norm_rope(q, k, qw, kw, cos, sin, interleaved=inter)
    for name, x, w, y in (("q", q, qw, qo), ("k", k, kw, ko)):
        check(name, y, *norm_rope_ref(x, w, cos, sin, P, 1e-6, d // 2, inter), dtype)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype,grad", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_backward(dtype, grad, d, inter):
    q, k, qw, kw, P, rn = _inputs(d, dtype, dtype.itemsize + 2 * grad.itemsize, 1, 8, 2)
    cos, sin = basp.rope_table(q.shape[1], d)
    print("backward", tuple(q.shape), dtype, grad, inter, flush=True)
    dy = rn(*q.shape, t=grad), rn(*k.shape, t=grad)
    dq, dk, dqw, dkw = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, interleaved=inter)
    for name, x, g, w, dx, dw in (("dq", q, dy[0], qw, dq, dqw), ("dk", k, dy[1], kw, dk, dkw)):
        rx, bx, rw, bw = norm_rope_bwd_ref(x, g, w, cos, sin, P, 1e-6, d, inter)
        check(name, dx, rx, bx, grad)
        check(name + "_weight", dw, rw, bw, F32)
        del rx, bx
