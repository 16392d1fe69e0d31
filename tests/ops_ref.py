"""Plain fp64 forms of the operators around attention, with bounds on a kernel's error (not
collected by pytest).

A rounding to a type is off by at most half a step: 2^-8 of the value in bf16, 2^-24 in fp32, 2^-4
in e4m3.  fp32 sums of n terms are off by at most n 2^-24 of the sum of magnitudes.  Each ``*_ref``
returns values and, beside them, the largest error that its formula allows."""
from __future__ import annotations

import math

import torch

F64 = torch.float64
U32, U16 = 2.0 ** -24, 2.0 ** -8   # half a step of fp32, of bf16
TINY = 2.0 ** -126


def half_step(dtype):
    return {torch.bfloat16: U16, torch.float32: U32}[dtype]


# --------------------------------------------------------- norm and rotation
def pair_columns(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(n, cos, sin, rot, interleaved):
    """(rotation of n, sum of the magnitudes added)."""
    a, b = pair_columns(rot, interleaved)
    y, mag = n.clone(), n.abs()
    y[..., a] = n[..., a] * cos - n[..., b] * sin
    y[..., b] = n[..., b] * cos + n[..., a] * sin
    mag = mag.clone()
    mag[..., a] = n[..., a].abs() * cos.abs() + n[..., b].abs() * sin.abs()
    mag[..., b] = n[..., b].abs() * cos.abs() + n[..., a].abs() * sin.abs()
    return y, mag


def angles(cos, sin, pos, rows):
    """cos, sin at int positions [b, S] as [b, S, 1, rot/2] (clamped; see where_bad)."""
    at = pos.long().clamp(0, max(rows - 1, 0))
    return cos.double()[at][:, :, None], sin.double()[at][:, :, None]


def norm_rope_ref(x, w, cos, sin, pos, eps, rot, interleaved):
    """(y, bound without the last rounding).  x [b, S, n, d], pos [b, S]."""
    X = x.double()
    if w is not None:
        r = 1 / torch.sqrt(X.pow(2).mean(-1, keepdim=True) + eps)
        X = X * r * w.double()
    mag = X.abs()
    if rot:
        X, mag = rotate(X, *angles(cos, sin, pos, cos.shape[0]), rot, interleaved)
        X = torch.where((pos >= cos.shape[0])[:, :, None, None], torch.nan, X)
    X = torch.where((pos < 0)[:, :, None, None], 0.0, X)
    # the mean: at most 24 roundings (products, sums, eps), halved by the root, whose own is one
    # step; r w, x r w; the rotation's products and sum
    return X, 32 * U32 * mag + TINY


def norm_rope_bwd_ref(x, dy, w, cos, sin, pos, eps, rot, interleaved):
    """(dx, bound without the last rounding, dw, bound)."""
    X, Z = x.double(), dy.double()
    dead = (pos < 0)[:, :, None, None]
    Z = torch.where(dead, 0.0, Z)
    zmag = Z.abs()
    if rot:
        c, s = angles(cos, sin, pos, cos.shape[0])
        Z, zmag = rotate(Z, c, -s, rot, interleaved)
        Z = torch.where((pos >= cos.shape[0])[:, :, None, None], torch.nan, Z)
    if w is None:
        return Z, 4 * U32 * zmag + TINY, None, None
    X = torch.where(dead, 1.0, X)
    W = w.double()
    d = X.shape[-1]
    r = 1 / torch.sqrt(X.pow(2).mean(-1, keepdim=True) + eps)
    g, gmag = Z * W, zmag * W.abs()
    k = r * r * (g * X).mean(-1, keepdim=True)
    kmag = r * r * (gmag * X.abs()).mean(-1, keepdim=True)
    dx = r * (g - X * k)
    dw = (Z * X * r).sum((0, 1, 2))
    rows = X.shape[0] * X.shape[1] * X.shape[2]
    chain = 64 + min(rows, 256) + rows // 1024   # additions on the longest path of the sum over rows
    return (dx, 64 * U32 * r * (gmag + X.abs() * kmag) + TINY, dw,
            (chain + 64) * U32 * (zmag * X.abs() * r).sum((0, 1, 2)) + TINY)


# ----------------------------------------------------------------- the cache
E_MIN = -110


def pow2(e):
    """2^e in fp64 for whole e, from its bits (pow and ldexp on the GPU are an ulp off for some)."""
    return ((e.long() + 1023) << 52).view(F64)


def quantise_ref(x):
    """(value that an 8-bit row holds, its scale byte) from the definition, by counting steps."""
    X = x.double()
    finite = X.isfinite()
    top = torch.where(finite, X.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.full_like(top, E_MIN)
    while True:
        up = top > 448 * pow2(e)
        if not up.any():
            break
        e = torch.where(up, e + 1, e)
    u = X * pow2(-e)
    exp = torch.frexp(torch.where(finite, u.abs().clamp(min=2.0 ** -6), 1.0))[1]
    step = pow2(exp - 4)
    v = torch.round(u / step) * step * pow2(e)
    # 2^128 is no bf16: the next smaller e4m3 value stands for it
    v = torch.where(v.abs() >= 2.0 ** 128, v.sign() * 240 * 2.0 ** 120, v)
    return torch.where(finite, v, torch.nan), (e[..., 0] + 127).to(torch.uint8)


def gather_ref(pages, scales, table, n):
    """The first n tokens of one sequence, [n, n_k, d] fp64; NaN on page numbers out of range."""
    n_pages, n_k, page, d = pages.shape
    out = torch.full((n, n_k, d), torch.nan, dtype=F64, device=pages.device)
    for p in range(-(-n // page)):
        m = min(page, n - p * page)
        i = int(table[p]) if p < table.numel() else -1
        if 0 <= i < n_pages:
            x = pages[i, :, :m].double()
            if scales is not None:
                x = x * pow2(scales[i, :, :m].int() - 127)[..., None]
            out[p * page:p * page + m] = x.transpose(0, 1)
    return out


def decode_ref(q, K, V, scale):
    """q [n_q, d] over K, V [n, n_k, d]: (O, bound of O without the last rounding, LSE, bound)."""
    n, n_k, d = K.shape
    n_q = q.shape[0]
    if n == 0:
        z = torch.zeros(n_q, d, dtype=F64, device=K.device)
        l = torch.full((n_q,), -math.inf, dtype=F64, device=K.device)
        return z, z, l, torch.zeros_like(l)
    rep = n_q // n_k
    Q = q.double().view(n_k, rep, d)
    Kt = K.permute(1, 2, 0).contiguous()
    s = torch.matmul(Q, Kt) * scale
    a = (torch.matmul(Q.abs(), Kt.abs()) * scale).amax(-1, keepdim=True)
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = torch.exp(s - lse)
    Vh = V.transpose(0, 1).contiguous()
    O, mag = torch.matmul(p, Vh), torch.matmul(p, Vh.abs())
    # a score: d products summed, then scaled (times log2 e); its error twice, in the weight and in the
    # sum of weights; the weight's rounding to bf16; the sums over keys in blocks of at most
    # 2^12 additions
    rel = 2 * (d + 16) * U32 * a + U16 + 2.0 ** -12
    lb = (d + 16) * U32 * a + 2.0 ** -12 * 1.0 / 16 + 8 * U32 * lse.abs()
    return (O.view(n_q, d), (rel * mag).view(n_q, d), lse.view(n_q), lb.view(n_q))


def check(name, got, ref, bound, dtype=None):
    """got against ref within bound plus the last rounding; not-a-number and infinities in the same
    places."""
    got = got.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    nan = ref.isnan()
    assert torch.equal(got.isnan(), nan), f"{name}: NaN in other places"
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf]), f"{name}: infinities differ"
    live = ~nan & ~inf
    tol = bound + (half_step(dtype) * (ref.abs() + bound) if dtype is not None else 0)
    off = (got - ref).abs()[live]
    if off.numel():
        worst = (off / tol[live].clamp(min=1e-300)).where(off > 0, torch.zeros_like(off)).max()
        print(f"  {name}: max|d| {off.max():.3e}, {worst:.3f} of the bound", flush=True)
        assert worst <= 1, f"{name}: {worst:.3f} of the allowed error (max {off.max():.3e})"
