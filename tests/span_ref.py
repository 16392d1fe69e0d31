"""Plain fp64 forms of attention over spans with bounds on a kernel's error (not collected by pytest).

Roundings are off by at most half a step (ops_ref): U16 = 2^-8 of the value in bf16, U32 = 2^-24 in
fp32.  A kernel's products take bf16 operands exactly, their fp32 sums of n terms are off by at most
n U32 of the sum of magnitudes, P and dS are rounded to bf16 once, and so are O and bf16 gradients."""
from __future__ import annotations

import math

import torch

from ops_ref import F64, TINY, U16, U32

EXP = 2.0 ** -20    # of the hardware's 2^x, with the roundings of its argument's last sum


def seen_of(spans, b, S, device):
    at = torch.arange(S, device=device)
    if spans is None:
        return (at <= at[:, None]).expand(b, S, S)
    lo, hi = spans.long().clamp(0, S)[..., None].unbind(2)
    return (at >= lo) & (at < hi)


def scores(q, k, scale, cap, slopes):
    """u [b, n_q, S, S], d u / d s, and the largest error of u, of the derivative (fp64)."""
    b, S, n_q, d = q.shape
    rep = n_q // k.shape[2]
    Q, K = q.double().transpose(1, 2), k.double().transpose(1, 2).repeat_interleave(rep, 1)
    Kt = K.transpose(2, 3).contiguous()
    s = torch.matmul(Q, Kt) * scale
    e = torch.matmul(Q.abs(), Kt.abs()) * scale * (d + 8) * U32
    one, e1 = torch.ones_like(s), torch.zeros_like(s)
    if cap:
        t = torch.tanh(s / cap)
        one = 1 - t * t
        # tanh from an exponential and a reciprocal: 2^-21 (the header), the scaled argument's
        # roundings 4 U32 |x| times the derivative, of which x (1 - tanh^2) stays below 0.5
        e = e * one + cap * (2.0 ** -21 + 2 * U32) + e * e / cap
        e1 = 2 * e / cap + 2.0 ** -20
        s = cap * t
    e = e + 6 * U32 * s.abs()
    if slopes is not None:
        at = torch.arange(S, device=q.device, dtype=F64)
        bias = slopes.double().view(-1, 1, 1) * (at[:, None] - at).abs()
        s = s - bias
        e = e + 6 * U32 * bias.abs()
    return s, one, e, e1


def fwd_ref(q, k, v, spans, scale, cap, slopes):
    """(O, bound without the last rounding, LSE, bound)."""
    b, S, n_q, d = q.shape
    rep = n_q // k.shape[2]
    u, _, e, _ = scores(q, k, scale, cap, slopes)
    seen = seen_of(spans, b, S, q.device)[:, None]
    u = u.masked_fill(~seen, -math.inf)
    e = e.masked_fill(~seen, 0)
    empty = ~seen.any(-1)
    lse = torch.logsumexp(u, -1)
    p = torch.exp(u - lse.masked_fill(empty, 0)[..., None])
    V = v.double().transpose(1, 2).repeat_interleave(rep, 1)
    n = seen.sum(-1, keepdim=True)
    worst = e.amax(-1, keepdim=True)
    O = torch.matmul(p, V)
    # a weight: rounded, its exponent, and the reference's; the row's sum alike but unrounded
    bound = torch.matmul(p * (U16 + 2 * EXP + (2 * n + 16) * U32 + e + worst), V.abs()) * 1.01
    if cap and cap <= 64:
        # With the fixed reference O is divided by the sum L' of weights of which some are rounded:
        # w_j = p_j (1 + d_j), |d_j| <= U16, so L' = L (1 + x) with |x| <= U16 sum p_j = U16, and
        # sum w_j v_j / L' - O = (sum p_j d_j v_j - x O) / (1 + x): U16 |O| more.
        bound = bound + U16 * 1.01 * O.abs()
    # weights below 2^-126 may be taken for 0: relative to the row's sum, which is 2^-8 at least with
    # a reference that follows the maximum to 2^8, and 2^(-1.45 cap) with the fixed one (cap <= 64)
    lost = 2.0 ** -116 if not cap or cap > 64 else 2.0 ** -33
    bound = bound + torch.matmul(seen.double() * lost, V.abs())
    top = u.masked_fill(~seen, 0).abs().amax(-1)
    el = worst[..., 0] + 2 * EXP + (n[..., 0] + 8) * U32 + 4 * U32 * (lse.masked_fill(empty, 0).abs()
                                                                      + top)
    return (O.transpose(1, 2), bound.transpose(1, 2) + TINY, lse, el * 1.01)


def bwd_ref(q, k, v, o, lse, do, spans, scale, cap, slopes):
    """((dQ, bound), (dK, bound), (dV, bound)) from these o and lse, without the last rounding."""
    b, S, n_q, d = q.shape
    n_k = k.shape[2]
    rep = n_q // n_k
    u, one, e, e1 = scores(q, k, scale, cap, slopes)
    seen = seen_of(spans, b, S, q.device)[:, None]
    L = lse.double()[..., None]
    L = L.masked_fill(L == -math.inf, 0)
    p = torch.exp((u - L).masked_fill(~seen, -math.inf))
    # the exponent's fp32 sums: of u, the LSE and, with slopes, the bias taken apart by rows and keys
    ep = e + EXP + 8 * U32 * (u.abs() + L.abs())
    if slopes is not None:
        ep = ep + 16 * U32 * 64 * slopes.double().abs().view(-1, 1, 1)
    heads = lambda x: x.double().transpose(1, 2)  # noqa: E731
    Q, dO, O = heads(q), heads(do), heads(o)
    K, V = (heads(x).repeat_interleave(rep, 1) for x in (k, v))
    dp = torch.matmul(dO, V.transpose(2, 3).contiguous())
    D = (dO * O).sum(-1, keepdim=True)
    g = dp - D
    eg = (d + 8) * U32 * (torch.matmul(dO.abs(), V.abs().transpose(2, 3).contiguous())
                          + (dO * O).abs().sum(-1, keepdim=True))
    ds = p * g * one
    eds = p * (one * (g.abs() * (U16 + ep + 4 * U32) + eg) + (g.abs() + eg) * e1)
    epv = p * (U16 + ep)
    # P, and P g, below 2^-126 may be taken for 0, which is off by that much: keys whose weights all
    # lie there (scores some 87 below a row's LSE) have no other error
    epv = epv + TINY
    eds = eds + TINY * (1 + g.abs())
    group = lambda x: x.view(b, n_k, rep, S, d).sum(2)  # noqa: E731
    t = lambda x: x.transpose(2, 3).contiguous()  # noqa: E731
    n = S + 16
    out = [(torch.matmul(ds, K) * scale,
            torch.matmul(eds + n * U32 * ds.abs(), K.abs()) * scale * 1.02)]
    out.append((group(torch.matmul(t(ds), Q)) * scale,
                group(torch.matmul(t(eds + rep * n * U32 * ds.abs()), Q.abs())) * scale * 1.02))
    out.append((group(torch.matmul(t(p), dO)),
                group(torch.matmul(t(epv + rep * n * U32 * p), dO.abs())) * 1.02))
    return tuple((x.transpose(1, 2), bound.transpose(1, 2) + TINY) for x, bound in out)


def documents(b, S, mean, prefix, pad, gen):
    """Random packed sequences: (documents [b, S], prefix [b, S]) on the CPU."""
    docs = torch.zeros(b, S, dtype=torch.int32)
    pre = torch.zeros(b, S, dtype=torch.int32)
    for s in range(b):
        at, i = 0, 0
        while at < S:
            n = int(torch.randint(1, 2 * mean + 1, (1,), generator=gen))
            docs[s, at:at + n] = i
            pre[s, at:at + n] = int(torch.randint(0, prefix + 1, (1,), generator=gen))
            at, i = at + n, i + 1
        if pad:
            docs[s, S - pad:] = -1
    return docs, pre


def wild_spans(b, S, gen):
    """Any numbers at all as spans: inside, outside, reversed, far past the ends."""
    lo = torch.randint(-S // 4 - 2, S + 1, (b, S), generator=gen)
    hi = lo + torch.randint(-S // 8 - 2, S + 2, (b, S), generator=gen)
    far = torch.rand(b, S, generator=gen)
    lo = torch.where(far < 0.02, -2 ** 31, lo)
    hi = torch.where((far > 0.01) & (far < 0.05), 2 ** 31 - 1, hi)
    return torch.stack((lo, hi), -1).to(torch.int32)
