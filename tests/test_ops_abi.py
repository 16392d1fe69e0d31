"""The C ABI and the binding of the operators around attention on a host without a GPU: every
documented refusal, before any HIP call (the pointers are fake: only invalid or empty calls)."""
import ctypes
import math

import pytest
import torch

import paper_2609_03151_amd as basp

OK, NULL, SHAPE, RANK, UNSUP, ALIGN, WS = range(7)
BF, F32, E4M3 = 0, 1, 2
vp = ctypes.c_void_p


def P(n):
    return [0x10000 * (i + 1) for i in range(n)]


def _with(base, **over):
    d = dict(base)
    assert set(over) <= set(d), over
    d.update(over)
    return d


NORM = dict(q=0x10000, k=0x20000, qo=0x30000, ko=0x40000, qw=0x50000, kw=0x60000, cos=0x70000,
            sin=0x80000, pos=None, b=2, S=8, n_q=4, n_k=2, d=128, rot=128, rows=8, q_row=512,
            k_row=256, qo_row=512, ko_row=256, eps=1e-6, pos0=0, inter=0, dtype=BF, stream=None)


@pytest.mark.parametrize("code,over", [
    (SHAPE, dict(b=-1)), (SHAPE, dict(S=-1)), (SHAPE, dict(n_q=0)), (SHAPE, dict(n_k=0)),
    (SHAPE, dict(rot=4)), (SHAPE, dict(rot=136)), (SHAPE, dict(rot=-8)), (SHAPE, dict(rows=7)),
    (SHAPE, dict(pos0=1)), (SHAPE, dict(pos0=-1)), (SHAPE, dict(pos0=2 ** 31 - 1)),
    (SHAPE, dict(q_row=511)), (SHAPE, dict(k_row=0)),
    (SHAPE, dict(qo_row=-512)), (SHAPE, dict(ko_row=255)), (SHAPE, dict(rows=-1)),
    (UNSUP, dict(d=72, rot=72)), (UNSUP, dict(d=256)), (UNSUP, dict(dtype=E4M3)),
    (UNSUP, dict(dtype=-1)), (UNSUP, dict(eps=-1e-6)), (UNSUP, dict(eps=math.nan)),
    (UNSUP, dict(eps=math.inf)), (UNSUP, dict(b=2 ** 16, S=2 ** 12, n_q=2, rows=2 ** 12)),
    (UNSUP, dict(b=2 ** 31 - 1, S=2 ** 31 - 1, n_k=2 ** 20, k_row=2 ** 27, rows=2 ** 31 - 1)),
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(qo=None)), (NULL, dict(ko=None)),
    (NULL, dict(qw=None)), (NULL, dict(kw=None)), (NULL, dict(cos=None)), (NULL, dict(sin=None)),
    (NULL, dict(cos=None, sin=None)), (NULL, dict(rot=0)),
    (ALIGN, dict(q=0x10004)), (ALIGN, dict(ko=0x40002)), (ALIGN, dict(dtype=F32, k=0x20008)),
    (ALIGN, dict(qw=0x50004)), (ALIGN, dict(sin=0x80008)), (ALIGN, dict(pos=0x90002)),
    (ALIGN, dict(q_row=514)), (ALIGN, dict(qo_row=513)),
    (OK, dict(b=0, q=None, cos=None, sin=None)), (OK, dict(S=0, rows=0, qo=None)),
])
def test_norm_rope_refuses(code, over):
    a = _with(NORM, **over)
    assert basp.lib().basp_qk_norm_rope(*a.values()) == code


NORM_BWD = dict(q=0x10000, k=0x20000, dqo=0x30000, dko=0x40000, dq=0x31000, dk=0x41000,
                qw=0x50000, kw=0x60000, dqw=0x51000, dkw=0x61000, cos=0x70000, sin=0x80000,
                pos=None, ws=0x90000, n=1 << 20, b=2, S=8, n_q=4, n_k=2, d=128, rot=128, rows=8,
                q_row=512, k_row=256, eps=1e-6, pos0=0, inter=0, dtype=BF, grad=F32, stream=None)


@pytest.mark.parametrize("code,over", [
    (SHAPE, dict(b=-1)), (SHAPE, dict(rot=12)), (SHAPE, dict(rows=7)), (SHAPE, dict(q_row=1)),
    (UNSUP, dict(d=48, rot=48)), (UNSUP, dict(grad=E4M3)), (UNSUP, dict(dtype=7)),
    (UNSUP, dict(b=2 ** 16, S=2 ** 12, n_q=2, rows=2 ** 12)),
    (NULL, dict(q=None)), (NULL, dict(dko=None)), (NULL, dict(dk=None)), (NULL, dict(dqw=None)),
    (NULL, dict(qw=None)), (NULL, dict(sin=None)), (NULL, dict(ws=None)),
    (ALIGN, dict(dq=0x31008)), (ALIGN, dict(grad=BF, dko=0x40004)), (ALIGN, dict(dkw=0x61002)),
    (ALIGN, dict(ws=0x90008)), (ALIGN, dict(k=0x20004)), (ALIGN, dict(k_row=258)),
    (WS, dict(n=0)), (OK, dict(b=0, q=None, ws=None, n=0)),
])
def test_norm_rope_bwd_refuses(code, over):
    a = _with(NORM_BWD, **over)
    assert basp.lib().basp_qk_norm_rope_bwd(*a.values()) == code


def test_norm_rope_bwd_workspace():
    f = basp.qk_norm_rope_bwd_workspace_bytes
    a = _with(NORM_BWD, n=f(2, 8, 4, 2, 128) - 1)
    assert basp.lib().basp_qk_norm_rope_bwd(*a.values()) == WS
    assert f(0, 8, 4, 2, 128) == f(2, 0, 4, 2, 128) == f(2, 8, 4, 2, 72) == f(-1, 8, 4, 2, 64) == 0
    assert f(2 ** 16, 2 ** 12, 2, 1, 64) == 0
    assert 0 < f(1, 1, 1, 1, 64) <= f(1, 2 ** 20, 8, 1, 64) <= 1 << 22


CACHE = dict(k=0x10000, v=0x20000, kp=0x30000, vp=0x40000, ks=None, vs=None, table=0x50000,
             start=0x60000, count=None, b=2, T=4, n_k=2, d=128, page=64, n_pages=10, max_pages=5,
             k_row=256, v_row=256, dtype=BF, stream=None)


@pytest.mark.parametrize("code,over", [
    (SHAPE, dict(b=-1)), (SHAPE, dict(T=-1)), (SHAPE, dict(n_k=0)), (SHAPE, dict(page=0)),
    (SHAPE, dict(n_pages=0)), (SHAPE, dict(max_pages=0)), (SHAPE, dict(k_row=255)),
    (SHAPE, dict(v_row=0)),
    (UNSUP, dict(d=100, k_row=1000, v_row=1000)), (UNSUP, dict(page=48)), (UNSUP, dict(page=8)),
    (UNSUP, dict(page=512)), (UNSUP, dict(dtype=F32)), (UNSUP, dict(dtype=3)),
    (UNSUP, dict(n_pages=2 ** 30, n_k=2)), (UNSUP, dict(b=2 ** 15, T=2 ** 13)),
    (NULL, dict(k=None)), (NULL, dict(vp=None)), (NULL, dict(table=None)),
    (NULL, dict(start=None)), (NULL, dict(dtype=E4M3)), (NULL, dict(dtype=E4M3, ks=0x70000)),
    (NULL, dict(ks=0x70000, vs=0x80000)),
    (ALIGN, dict(k=0x10008)), (ALIGN, dict(vp=0x40008)), (ALIGN, dict(table=0x50002)),
    (ALIGN, dict(count=0x90001)), (ALIGN, dict(k_row=260)),
    (ALIGN, dict(dtype=E4M3, ks=0x70002, vs=0x80000)),
    (OK, dict(b=0, k=None, kp=None)), (OK, dict(T=0, table=None)),
])
def test_kv_write_refuses(code, over):
    a = _with(CACHE, **over)
    L = basp.lib()
    assert L.basp_kv_write(*a.values()) == code
    if "k_row" in over or "v_row" in over or over == dict(start=None):
        return   # the read has no strides, and may start at 0
    r = [a[n] for n in ("kp", "vp", "ks", "vs", "table", "start", "count", "k", "v", "b", "T",
                        "n_k", "d", "page", "n_pages", "max_pages", "dtype", "stream")]
    assert L.basp_kv_read(*r) == code


DECODE = dict(q=0x10000, kp=0x30000, vp=0x40000, ks=None, vs=None, table=0x50000, lens=0x60000,
              o=0x70000, lse=None, ws=0x80000, n=1 << 30, b=2, n_q=8, n_k=2, d=128, page=64,
              n_pages=10, max_pages=500, max_len=32000, q_row=1024, scale=0.1, dtype=BF,
              stream=None)


@pytest.mark.parametrize("code,over", [
    (SHAPE, dict(b=-1)), (SHAPE, dict(n_q=7)), (SHAPE, dict(n_q=0)), (SHAPE, dict(max_len=0)),
    (SHAPE, dict(n_pages=0)), (SHAPE, dict(q_row=1023)),
    (UNSUP, dict(d=72)), (UNSUP, dict(page=17)), (UNSUP, dict(dtype=F32)),
    (UNSUP, dict(scale=0.0)), (UNSUP, dict(scale=-1.0)), (UNSUP, dict(scale=math.nan)),
    (UNSUP, dict(scale=math.inf)), (UNSUP, dict(b=2 ** 19)), (UNSUP, dict(max_len=2 ** 30 + 1)),
    (UNSUP, dict(n_pages=2 ** 30)),
    (NULL, dict(q=None)), (NULL, dict(kp=None)), (NULL, dict(lens=None)), (NULL, dict(o=None)),
    (NULL, dict(table=None)), (NULL, dict(dtype=E4M3)), (NULL, dict(ws=None)),
    (ALIGN, dict(q=0x10008)), (ALIGN, dict(o=0x70004)), (ALIGN, dict(lse=0x90002)),
    (ALIGN, dict(lens=0x60001)), (ALIGN, dict(q_row=1028)), (ALIGN, dict(ws=0x80008)),
    (WS, dict(n=16)), (OK, dict(b=0, q=None, lens=None)),
])
def test_attn_decode_refuses(code, over):
    a = _with(DECODE, **over)
    assert basp.lib().basp_attn_decode(*a.values()) == code


def test_attn_decode_workspace():
    f = basp.attn_decode_workspace_bytes
    need = f(2, 8, 2, 128, 32000)
    a = _with(DECODE, n=need - 1)
    assert basp.lib().basp_attn_decode(*a.values()) == WS
    assert f(0, 8, 2, 128, 1000) == f(2, 7, 2, 128, 1000) == f(2, 8, 2, 72, 1000) == 0
    assert f(2, 8, 2, 128, 0) == f(2, 8, 2, 128, -5) == 0
    # a launch's workgroups stay a 32-bit count of threads whatever the lengths
    for b, n_q, L in ((1, 1, 2 ** 30), (2 ** 21, 1, 2 ** 30), (2 ** 18, 15, 2 ** 20)):
        assert f(b, n_q, 1, 64, L) // (66 * 4) * 256 < 2 ** 32


def test_binding_refuses():
    """Wrong types, shapes and layouts raise before anything is launched."""
    t = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):    # a host tensor
        basp.qk_norm_rope(t, t, None, None, None, None)
    with pytest.raises(ValueError):   # q and k disagree
        basp.qk_norm_rope(t, t[:, :3], None, None, None, None)
    with pytest.raises(ValueError):   # cos without sin
        basp.qk_norm_rope(t, t, None, None, torch.zeros(4, 32), None)
    with pytest.raises(ValueError):
        basp.qk_norm_rope(t, t, torch.ones(64), None, None, None)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(TypeError):
        basp.kv_write(t, t, torch.zeros(1, 2, 16, 64, dtype=torch.float16),
                      torch.zeros(1, 2, 16, 64, dtype=torch.float16), i, i[0])
    with pytest.raises(ValueError):   # an 8-bit cache without scales
        basp.attn_decode(t[0], torch.zeros(1, 2, 16, 64, dtype=torch.float8_e4m3fn),
                         torch.zeros(1, 2, 16, 64, dtype=torch.float8_e4m3fn), i, i[0])
    with pytest.raises(ValueError):
        basp.attn_decode(t, t, t, i, i[0])


def test_rope_table():
    cos, sin = basp.rope_table(200000, 64, base=500000.0, device="cpu")
    assert cos.shape == sin.shape == (200000, 32) and cos.dtype == torch.float32
    p, i = 199999, 3
    a = p * 500000.0 ** (-2 * i / 64)
    assert abs(cos[p, i].item() - math.cos(a)) < 1e-6 and abs(sin[p, i].item() - math.sin(a)) < 1e-6


def test_attn_decode_counts_in_32_bits():
    """Units of keys of all heads, and workgroups on top in the division that deals them out, are
    32-bit counts on the device."""
    f = basp.attn_decode_workspace_bytes
    assert f(2 ** 22 - 1, 1, 1, 64, 65536) == 0 == f(2 ** 15, 1, 1, 64, 2 ** 22)
    assert f(2 ** 15 - 1, 1, 1, 64, 2 ** 22) > 0
