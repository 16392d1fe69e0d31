"""The C ABI and the binding of attention over spans on a host without a GPU: every documented refusal,
before any HIP call (the pointers are fake: only invalid or empty calls)."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp

OK, NULL, SHAPE, RANK, UNSUP, ALIGN, WS = range(7)
BF, F32, E4M3 = 0, 1, 2
BIG = 2 ** 31 - 1


def _with(base, **over):
    d = dict(base)
    assert set(over) <= set(d), over
    d.update(over)
    return d


SIZES = dict(b=2, S=8, n_q=4, n_k=2, d=128, q_row=512, k_row=256, v_row=256, scale=0.1, cap=0.0)
FWD = dict(q=0x10000, k=0x20000, v=0x30000, spans=0x40000, slopes=0x50000, o=0x60000, lse=0x70000,
           **SIZES, stream=None)
BWD = dict(q=0x10000, k=0x20000, v=0x30000, spans=0x40000, slopes=0x50000, o=0x60000, lse=0x70000,
           d_o=0x80000, dq=0x90000, dk=0xA0000, dv=0xB0000, ws=0xC0000, n=1 << 30, **SIZES,
           grad=F32, stream=None)
SHARED = [
    (SHAPE, dict(b=-1)), (SHAPE, dict(S=-1)), (SHAPE, dict(n_q=0)), (SHAPE, dict(n_k=0)),
    (SHAPE, dict(n_k=3)), (SHAPE, dict(n_k=8)), (SHAPE, dict(d=0)), (SHAPE, dict(q_row=511)),
    (SHAPE, dict(k_row=0)), (SHAPE, dict(v_row=-256)),
    (UNSUP, dict(d=72)), (UNSUP, dict(d=256, q_row=1024, k_row=512, v_row=512)),
    (UNSUP, dict(scale=0.0)), (UNSUP, dict(scale=-1.0)), (UNSUP, dict(scale=math.nan)),
    (UNSUP, dict(scale=math.inf)), (UNSUP, dict(cap=-1.0)), (UNSUP, dict(cap=math.nan)),
    (UNSUP, dict(cap=1025.0)), (UNSUP, dict(cap=math.inf)),
    (UNSUP, dict(cap=1e-38, scale=1e30)),
    (UNSUP, dict(b=65536)), (UNSUP, dict(b=2 ** 15, S=2 ** 12)), (UNSUP, dict(b=60000, S=1, n_q=64,
                                                                              q_row=8192)),
    (UNSUP, dict(b=1, S=BIG)), (UNSUP, dict(b=1, S=2 ** 21)), (UNSUP, dict(q_row=2 ** 40)),
    (UNSUP, dict(v_row=2 ** 23)), (UNSUP, dict(k_row=2 ** 62)),
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(o=None)),
    (NULL, dict(lse=None)),
    (ALIGN, dict(q=0x10008)), (ALIGN, dict(k=0x20002)), (ALIGN, dict(v=0x30008)),
    (ALIGN, dict(spans=0x40004)), (ALIGN, dict(slopes=0x50002)), (ALIGN, dict(o=0x60008)),
    (ALIGN, dict(lse=0x70002)), (ALIGN, dict(q_row=516)), (ALIGN, dict(k_row=260)),
    (ALIGN, dict(v_row=257)),
    (OK, dict(b=0, q=None, spans=None)), (OK, dict(S=0, o=None, lse=None)),
]


@pytest.mark.parametrize("code,over", SHARED)
def test_fwd_refuses(code, over):
    assert basp.lib().basp_attn_span_fwd(*_with(FWD, **over).values()) == code


@pytest.mark.parametrize("code,over", SHARED + [
    (UNSUP, dict(grad=E4M3)), (UNSUP, dict(grad=-1)),
    (NULL, dict(d_o=None)), (NULL, dict(dq=None)), (NULL, dict(dk=None)), (NULL, dict(dv=None)),
    (NULL, dict(ws=None)), (ALIGN, dict(d_o=0x80008)), (ALIGN, dict(dq=0x90004)),
    (ALIGN, dict(dk=0xA0008)), (ALIGN, dict(dv=0xB0002)), (ALIGN, dict(ws=0xC0008)),
    (WS, dict(n=0)), (WS, dict(n=1000)),
    # more workgroups than a launch holds
    (UNSUP, dict(b=100, S=131072, n_q=8, n_k=8, d=64, q_row=512, k_row=512, v_row=512)),
])
def test_bwd_refuses(code, over):
    assert basp.lib().basp_attn_span_bwd(*_with(BWD, **over).values()) == code


def test_workspace():
    need = basp.attn_span_bwd_workspace_bytes
    for bad in ((0, 8, 4, 2, 128), (1, 0, 4, 2, 128), (1, 8, 4, 3, 128), (1, 8, 4, 2, 100),
                (-1, 8, 4, 2, 128), (1, BIG, 4, 2, 128)):
        assert need(*bad) == 0
    # -LSE and -D of padded rows, their spans, one partial sum
    assert 64 * 4 * 8 <= need(1, 8, 4, 2, 128) < 64 * 1024
    # at most 16 sums of each of dK and dV up to 1M rows, and what each row keeps
    S, n_q, n_k, d = 1 << 17, 8, 1, 128
    assert need(1, S, n_q, n_k, d) <= 16 * 2 * S * n_k * d * 4 * n_q + 64 * S * n_q


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_binding_refuses():
    q, k = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 1, 64,
                                                                       dtype=torch.bfloat16)
    spans = torch.zeros(1, 4, 2, dtype=torch.int32)
    with pytest.raises(TypeError):       # host tensors
        basp.attn_span_fwd(q, k, k, spans)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q[0], k, k, spans)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q, k[:, :3], k, spans)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q, k, k[:, :3], spans)
    with pytest.raises(TypeError):
        basp.attn_span_fwd(q, k, k.float(), spans)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q, k, k, spans[:, :, :1])
    with pytest.raises(TypeError):
        basp.attn_span_fwd(q, k, k, spans.long())
    with pytest.raises(ValueError):      # a cap of 0 is no cap
        basp.attn_span_fwd(q, k, k, spans, cap=0.0)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q, k, k, spans, cap=-3.0)
    with pytest.raises(ValueError):
        basp.attn_span_fwd(q, k, k, spans, slopes=torch.zeros(3))
    with pytest.raises(ValueError):      # every other element of a head
        basp.attn_span_fwd(torch.zeros(1, 4, 2, 128, dtype=torch.bfloat16)[..., ::2], k, k, spans)
    lse = torch.zeros(1, 2, 4)
    with pytest.raises(TypeError):
        basp.attn_span_bwd(q, k, k, q, lse, q, spans, grad_dtype=torch.float16)
    with pytest.raises(ValueError):
        basp.attn_span_bwd(q, k, k, q, lse[:, :1], q, spans)


def test_attn_spans():
    docs = torch.tensor([[0, 0, 0, 1, 1, -1], [4, 4, 4, 4, 4, 4], [-1, -1, 7, 7, -2, 7]])
    assert basp.attn_spans(docs).tolist() == [
        [[0, 1], [0, 2], [0, 3], [3, 4], [3, 5], [0, 0]], [[0, i + 1] for i in range(6)],
        [[0, 0], [0, 0], [2, 3], [2, 4], [0, 0], [5, 6]]]
    pre = torch.tensor([[2, 2, 2, 9, 9, 9], [0] * 6, [1] * 6])
    got = basp.attn_spans(docs, pre)
    assert got.dtype == torch.int32 and got.is_contiguous()
    assert got[0].tolist() == [[0, 2], [0, 2], [0, 3], [3, 5], [3, 5], [0, 0]]
    assert torch.equal(got[1:], basp.attn_spans(docs)[1:])
    with pytest.raises(ValueError):
        basp.attn_spans(docs[0])
    with pytest.raises(ValueError):
        basp.attn_spans(docs, pre[:2])
    assert basp.attn_spans(docs[:, :0]).shape == (3, 0, 2)
