"""The C ABI and the binding of attn_decode_shared on a host without a GPU: every documented refusal,
before any HIP call (the pointers are fake: only invalid or empty calls)."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp

OK, NULL, SHAPE, RANK, UNSUP, ALIGN, WS = range(7)
BF, F32, E4M3 = 0, 1, 2
CALL = dict(q=0x10000, k=0x20000, v=0x30000, ks=None, vs=None, table=0x40000, lens=0x50000,
            groups=0x60000, prefix=0x70000, slopes=0x80000, o=0x90000, lse=0xA0000, ws=0xB0000,
            n=1 << 40, b=2, n_q=4, n_k=2, d=128, page=64, n_pages=10, max_pages=4, max_len=256,
            n_groups=1, q_row=512, scale=0.1, cap=0.0, dtype=BF, stream=None)


@pytest.mark.parametrize("code,over", [
    (SHAPE, dict(b=-1)), (SHAPE, dict(n_q=3)), (SHAPE, dict(n_k=0)), (SHAPE, dict(max_len=0)),
    (SHAPE, dict(page=0)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(max_pages=0)),
    (SHAPE, dict(q_row=511)), (SHAPE, dict(n_groups=-1)),
    (UNSUP, dict(d=72)), (UNSUP, dict(page=24)), (UNSUP, dict(dtype=F32)),
    (UNSUP, dict(scale=0.0)), (UNSUP, dict(scale=math.nan)), (UNSUP, dict(cap=-1.0)),
    (UNSUP, dict(cap=math.nan)), (UNSUP, dict(cap=1025.0)), (UNSUP, dict(cap=1e-38, scale=1e30)),
    (UNSUP, dict(n_groups=1 << 22)), (UNSUP, dict(b=1 << 21)), (UNSUP, dict(max_len=(1 << 30) + 1)),
    (UNSUP, dict(b=1 << 15, max_len=1 << 20)), (UNSUP, dict(n_pages=1 << 30)),
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(table=None)),
    (NULL, dict(lens=None)), (NULL, dict(o=None)), (NULL, dict(groups=None)),
    (NULL, dict(prefix=None)), (NULL, dict(ws=None)), (NULL, dict(ks=0x1000)),
    (NULL, dict(dtype=E4M3)),
    (ALIGN, dict(q=0x10008)), (ALIGN, dict(k=0x20008)), (ALIGN, dict(groups=0x60002)),
    (ALIGN, dict(prefix=0x70001)), (ALIGN, dict(slopes=0x80002)), (ALIGN, dict(o=0x90004)),
    (ALIGN, dict(lse=0xA0002)), (ALIGN, dict(ws=0xB0008)), (ALIGN, dict(q_row=516)),
    (WS, dict(n=0)), (WS, dict(n=1000)),
    (OK, dict(b=0, q=None, groups=None)),
])
def test_refuses(code, over):
    a = dict(CALL)
    assert set(over) <= set(a)
    a.update(over)
    assert basp.lib().basp_attn_decode_shared(*a.values()) == code


def test_workspace():
    need = basp.attn_decode_shared_workspace_bytes
    assert need(0, 4, 2, 128, 256, 1) == 0 and need(2, 4, 2, 128, 256, -1) == 0
    assert need(2, 4, 3, 128, 256, 1) == 0 and need(2, 4, 2, 100, 256, 1) == 0
    # no more than attn_decode's where nothing can be shared, but for the plan
    own = basp.attn_decode_workspace_bytes(64, 8, 2, 128, 32768)
    assert 0 < need(64, 8, 2, 128, 32768, 0) <= own + 64 * 1024
    assert need(1, 8, 2, 128, 32768, 1) <= basp.attn_decode_workspace_bytes(
        1, 8, 2, 128, 32768) + 64 * 1024
    # a partial result of 64 rows for each of about 512 workgroups at most, and a row's own
    assert need(64, 8, 2, 128, 32768, 4) <= own + 520 * 64 * 130 * 4 + 64 * 8 * 130 * 4 + 128 * 1024


def test_binding_refuses():
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    pages = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    table, lens = torch.zeros(2, 1, dtype=torch.int32), i32(1, 1)
    call = lambda *a, **k: basp.attn_decode_shared(q, pages, pages, table, lens, *a, **k)  # noqa: E731
    with pytest.raises(TypeError):       # host tensors
        call(i32(0, 2), i32(5))
    for a in ((None, i32(5)), (i32(0, 2), None), (i32(0, 2), i32(5, 6)), (i32(0, 1, 2), i32(5)),
              (i32(0, 2), torch.zeros(1, 1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call(*a)
    with pytest.raises(TypeError):
        call(i32(0, 2).long(), i32(5))
    for cap in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError):
            call(cap=cap)
    with pytest.raises(ValueError):
        call(slopes=torch.zeros(3))
    with pytest.raises(ValueError):
        basp.attn_decode_shared(q[:, :, :32], pages, pages, table, lens)
