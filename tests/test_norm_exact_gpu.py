"""Gradients of the norm's weights where every step is exact: rows of +1 and -1 have a norm of 1, quarter
turns permute and change signs, and sums of whole numbers below 2^24 have no rounding, so that a row
that is lost or added twice shows, however many there are."""
import pytest
import torch

import paper_2609_03151_amd as basp

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.mark.parametrize("dtype,grad", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("b,S,n_q,n_k,d,inter", [
    (1, 1, 1, 1, 64, False), (2, 37, 7, 1, 80, True), (1, 1024, 8, 8, 96, False),
    (3, 5461, 5, 2, 128, False), (1, 4096, 4, 4, 64, True), (1, 65537, 8, 1, 128, True),
    (2, 50001, 7, 2, 64, False), (1, 40003, 8, 2, 80, False), (1, 40003, 8, 2, 96, True)])
def test_weight_gradients_count_every_row(b, S, n_q, n_k, d, inter, dtype, grad):
    g = torch.Generator("cuda").manual_seed(S)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda")  # noqa: E731
    cos = (torch.arange(S, device="cuda") % 2).float()[:, None].expand(S, d // 2).contiguous()
    sin = 1 - cos
    print("case", b, S, n_q, n_k, d, inter, dtype, grad, flush=True)
    x, dy, want = [], [], []
    for n in (n_q, n_k):
        x.append((2 * ints(0, 2, b, S, n, d) - 1).to(dtype))
        dy.append(ints(-8, 9, b, S, n, d).to(grad))
        a, c = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, d // 2), slice(d // 2, d))
        z, y = torch.empty(b, S, n, d, dtype=F64, device="cuda"), dy[-1].double()
        C, T = cos.double()[:, None], sin.double()[:, None]
        z[..., a], z[..., c] = y[..., a] * C + y[..., c] * T, y[..., c] * C - y[..., a] * T
        want.append((z * x[-1].double()).sum((0, 1, 2)))
        assert 8 * b * S * n < 2 ** 24
    w = [2.0 ** ints(-1, 2, d).float() for _ in range(2)]
    _, _, dqw, dkw = basp.qk_norm_rope_bwd(*x, *dy, *w, cos, sin, eps=0.0, interleaved=inter)
    assert torch.equal(dqw.double(), want[0]) and torch.equal(dkw.double(), want[1])
