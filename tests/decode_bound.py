"""Attention of one token in fp64 with a bound that has no room for a weight rounded to one bf16, and
values that tell every run of 128 keys from every other (not collected by pytest).

The kernel's errors, for scores s_j = scale q . k_j, a_j = scale |q| . |k_j|, weights p_j:
  scores: d products added in fp32 (a step of 2^-23 each: an adder may truncate), the scale, its
    conversion to powers of two, and a difference to the running maximum, which is of size max a
    at most; a weight's relative error is its score's absolute one;
  weights: exp2 to a step; as two bf16, each off by at most 2^-8 of what it stands for: 2^-16;
  sums: per block of 32 keys two products of 32 terms, four steps for the rescaling (its factor and
    the multiplication); the four waves and the partial results are joined by a few more.
Sums of weights have the sums' steps and the weights' errors, not those of the two bf16."""
from __future__ import annotations

import math

import torch

from ops_ref import F64, TINY

STEP = 2.0 ** -23
UNIT = 128   # keys of a unit, the least that a workgroup takes


def additions(lens, n_q, n_k, max_len):
    """The most steps on the way of one weight to the result: the cut of a call, 768 workgroups (512
    where a kv head has more than 16 query heads), each a run of ceil(units / workgroups)."""
    rep = n_q // n_k
    rows, most = (16, 768) if rep <= 16 else (32, 512)
    per = n_k * -(-rep // rows)
    units = [-(-n // UNIT) if 0 < n <= max_len else 0 for n in lens]
    groups = min(most, per * len(lens) * -(-max_len // UNIT))
    quota = -(-per * sum(units) // groups)
    return 68 * quota + 2 * -(-max(units) // 8) + 40


def decode_exact(q, K, V, lens, scale, max_len=None):
    """q [b, n_q, d], K and V [b, T, n_k, d] (what the cache stands for), lengths <= T: (O, its bound
    without the last rounding, LSE, its bound)."""
    b, n_q, d = q.shape
    T, n_k = K.shape[1:3]
    chain = additions(lens, n_q, n_k, max_len or T)
    dead = torch.arange(T, device=K.device) >= torch.tensor(lens, device=K.device)[:, None]
    Q = q.double().view(b, n_k, n_q // n_k, d)
    Kt = K.double().masked_fill(dead[:, :, None, None], 0.0).permute(0, 2, 3, 1).contiguous()
    Vh = V.double().masked_fill(dead[:, :, None, None], 0.0).transpose(1, 2).contiguous()
    dead = dead[:, None, None]
    s = (torch.matmul(Q, Kt) * scale).masked_fill(dead, -math.inf)
    a = (torch.matmul(Q.abs(), Kt.abs()) * scale).masked_fill(dead, 0.0)
    top = a.amax(-1, keepdim=True)
    lse = torch.logsumexp(s, -1, keepdim=True)
    empty = lse == -math.inf
    p = torch.exp(s - lse.masked_fill(empty, 0.0))
    off = p * STEP * ((d + 8) * a + 8 * top + 2)   # of a weight
    O, mag = torch.matmul(p, Vh), torch.matmul(p, Vh.abs())
    off_sum = off.sum(-1, keepdim=True)
    bo = (torch.matmul(off, Vh.abs()) + (2.0 ** -16 + (chain + 8) * STEP) * mag
          + O.abs() * (off_sum + chain * STEP))
    n = torch.tensor(lens, device=K.device, dtype=F64).clamp(min=1).view(-1, 1, 1, 1)
    bl = off_sum + chain * STEP + 4 * STEP * (lse.masked_fill(empty, 0.0).abs() + n.log() + 1)
    # errors of second order: no weight is off by more than 2^-7
    assert not off.numel() or (off / p.clamp(min=1e-300)).max() < 2.0 ** -7
    up = 1 + 2.0 ** -6
    return (O.reshape(b, n_q, d), up * bo.reshape(b, n_q, d) + TINY, lse.reshape(b, n_q),
            up * bl.reshape(b, n_q))


def unit_values(b, T, n_k, d, device):
    """V in which 128 keys share one column that their neighbours leave at 0, another one for each head,
    and keys of the same column differ in size: a unit that is lost, taken twice or put in the
    place of another moves a column of O by a hundredth of it or more.  All are exact in 8 bits."""
    u = (torch.arange(T, device=device) // UNIT)[None, :, None]
    h = torch.arange(n_k, device=device)
    s = torch.arange(b, device=device)[:, None, None]
    col = ((u + 5 * h + 11 * s) % d)[..., None]
    V = torch.zeros(b, T, n_k, d, device=device)
    size = (1 + 0.25 * (u // d % 9) + 0 * col[..., 0]).float()
    return V.scatter_(3, col, size[..., None]).to(torch.bfloat16)
