"""Attention over spans, forward and backward, against plain fp64."""
import math

import pytest
import torch

import paper_2609_03151_amd as basp
import span_ref
from ops_ref import F64, check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _slopes(n):
    return 2.0 ** (-8.0 * torch.arange(1, n + 1, dtype=F32, device="cuda") / n)


def _inputs(b, S, n_q, n_k, d, seed, fused=False):
    g = torch.Generator("cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    if fused:
        qkv = rn(b, S, n_q + 2 * n_k, d)
        q, k, v = qkv[:, :, :n_q], qkv[:, :, n_q:n_q + n_k], qkv[:, :, n_q + n_k:]
    else:
        q, k, v = 2 * rn(b, S, n_q, d), rn(b, S, n_k, d), rn(b, S, n_k, d)
    return q, k, v, rn(b, S, n_q, d)


def _spans(kind, b, S, seed):
    gen = torch.Generator().manual_seed(seed)
    if kind == "causal":
        return None
    if kind == "wild":
        return span_ref.wild_spans(b, S, gen).cuda()
    if kind == "all":
        return torch.tensor([0, S], dtype=torch.int32).expand(b, S, 2).contiguous().cuda()
    mean, prefix, pad = {"docs": (max(1, S // 3), 0, 0), "prefix": (max(1, S // 2), S // 3, 0),
                         "short": (7, 3, min(S // 4, 70)), "one": (1, 0, 0)}[kind]
    docs, pre = span_ref.documents(b, S, mean, prefix, pad, gen)
    return basp.attn_spans(docs.cuda(), pre.cuda())


def _both(q, k, v, do, spans, scale, cap, slopes, grads=(BF16, F32)):
    print(f"case {tuple(q.shape)} {tuple(k.shape)} cap {cap} slopes {slopes is not None}", flush=True)
    o, lse = basp.attn_span_fwd(q, k, v, spans, scale=scale, cap=cap, slopes=slopes)
    assert o.dtype == BF16 and o.is_contiguous() and lse.dtype == F32
    O, bo, L, bl = span_ref.fwd_ref(q, k, v, spans, scale, cap, slopes)
    check("o", o, O, bo, BF16)
    check("lse", lse, L, bl, F32)
    ref = span_ref.bwd_ref(q, k, v, o, lse, do, spans, scale, cap, slopes)
    for dtype in grads:
        got = basp.attn_span_bwd(q, k, v, o, lse, do, spans, scale=scale, cap=cap, slopes=slopes,
                                 grad_dtype=dtype)
        for name, x, (r, bound) in zip(("dq", "dk", "dv"), got, ref):
            assert x.dtype == dtype and x.is_contiguous()
            check(f"{name} {dtype}", x, r, bound, dtype)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("cap", [None, 5.0, 50.0, 300.0])
@pytest.mark.parametrize("bias", [False, True])
def test_dims_and_rules(d, cap, bias):
    q, k, v, do = _inputs(2, 333, 4, 2, d, seed=d)
    _both(q, k, v, do, _spans("prefix", 2, 333, d), d ** -0.5, cap, _slopes(4) if bias else None)


@pytest.mark.parametrize("kind", ["causal", "docs", "prefix", "short", "one", "wild", "all"])
@pytest.mark.parametrize("S", [1, 2, 31, 64, 129, 777])
@pytest.mark.parametrize("rule", ["plain", "capped and biased"])
def test_spans_and_lengths(kind, S, rule):
    q, k, v, do = _inputs(2, S, 7, 1, 64 if S == 129 else 128, seed=S, fused=S % 2 == 1)
    cap, slopes = (None, None) if rule == "plain" else (20.0, _slopes(7))
    _both(q, k, v, do, _spans(kind, 2, S, 11 * S), 0.1, cap, slopes, grads=(F32,))


# fewer and more rows than fill the GPU: 64, 128 and 256 rows a workgroup, one and several partial
# sums of dK and dV
@pytest.mark.parametrize("b,S,n_q,n_k,d", [(1, 5000, 1, 1, 128), (2, 3001, 8, 2, 80),
                                           (1, 2311, 32, 4, 128), (3, 1100, 24, 8, 64),
                                           (40, 130, 16, 4, 96), (1, 4500, 4, 1, 96)])
@pytest.mark.parametrize("kind", ["causal", "docs", "wild"])
@pytest.mark.parametrize("cap", [None, 30.0])
def test_sizes(b, S, n_q, n_k, d, kind, cap):
    q, k, v, do = _inputs(b, S, n_q, n_k, d, seed=S)
    slopes = _slopes(n_q) if kind != "causal" else None
    _both(q, k, v, do, _spans(kind, b, S, S), d ** -0.5, cap, slopes, grads=(BF16,))


def test_slopes_of_any_sign():
    """Growing with distance, zero, and so steep that a row sees little but its nearest key."""
    q, k, v, do = _inputs(1, 400, 4, 4, 128, seed=3)
    slopes = torch.tensor([-0.05, 0.0, 40.0, 0.5], device="cuda")
    for kind in ("causal", "all", "wild"):
        for cap in (None, 10.0, 100.0):
            _both(q, k, v, do, _spans(kind, 1, 400, 5), 0.1, cap, slopes, grads=(F32,))


@pytest.mark.parametrize("cap", [None, 15.0, 100.0])
def test_gradient_against_differences(cap):
    """Directional derivatives of sum(O dO) in fp64 on the reference, central differences; the
    kernel's gradients are held to the reference's above."""
    q, k, v, do = _inputs(1, 70, 2, 1, 64, seed=8)
    spans, slopes = _spans("prefix", 1, 70, 4), _slopes(2)
    q, k, v = (x.double() for x in (q, k, v))
    O, _, L, _ = span_ref.fwd_ref(q, k, v, spans, 0.2, cap, slopes)
    ref = span_ref.bwd_ref(q, k, v, O, L, do, spans, 0.2, cap, slopes)
    g = torch.Generator("cuda").manual_seed(1)
    for i, (r, _) in enumerate(ref):
        way = torch.randn(r.shape, generator=g, device="cuda", dtype=F64)
        h, sides = 1e-5, []
        for s in (h, -h):
            x = [q, k, v]
            x[i] = x[i] + s * way
            sides.append((span_ref.fwd_ref(*x, spans, 0.2, cap, slopes)[0] * do.double()).sum())
        want = (sides[0] - sides[1]) / (2 * h)
        # the third derivative's term, h^2 times what is of order 10^3 here, and cancellation
        assert abs(want - (r * way).sum()) <= 1e-5 * (r * way).abs().sum()


def test_causal_is_attn_fwd():
    """Without a cap, slopes or spans: the causal attention, to the bounds of both."""
    q, k, v, do = _inputs(2, 1000, 8, 2, 128, seed=2)
    o, lse = basp.attn_span_fwd(q, k, v, None)
    o2, lse2 = basp.attn_fwd(q, k, v, G=1)
    _, bound, _, bl = span_ref.fwd_ref(q, k, v, None, 128 ** -0.5, None, None)
    assert ((o.double() - o2.double()).abs() <= 2 * bound + 2.0 ** -7 * o.double().abs()).all()
    assert ((lse - lse2).abs() <= 2 * bl + 1e-6).all()


def test_scores_far_apart():
    """Scores that grow along the row by hundreds of powers of two, and fall."""
    q, k, v, do = _inputs(1, 600, 2, 1, 64, seed=6)
    ramp = torch.linspace(-40, 40, 600, device="cuda")
    for sign in (1, -1):
        k2 = (k.float() * 0.1 + sign * ramp.view(1, -1, 1, 1) / 8).to(BF16)
        q2 = (q.float() * 0.1 + 1).to(BF16)
        for kind in ("causal", "wild"):
            _both(q2, k2, v, do, _spans(kind, 1, 600, 9), 1.0, None, None, grads=(F32,))
            _both(q2, k2, v, do, _spans(kind, 1, 600, 9), 1.0, 64.0, None, grads=(F32,))
            _both(q2, k2, v, do, _spans(kind, 1, 600, 9), 1.0, 1000.0, _slopes(2), grads=(F32,))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("cap", [None, 30.0])
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_values_do_not_count(bad, cap, d):
    """Rows of Q, K, V and dO that meet nothing may hold anything: a document of garbage between
    two, and padding."""
    b, S, n = 2, 300, 4
    q, k, v, do = _inputs(b, S, n, 2, d, seed=12)
    docs = torch.zeros(b, S, dtype=torch.int32)
    docs[:, 100:] = 1
    docs[:, 133:] = 2
    docs[1, 250:] = -1
    spans = basp.attn_spans(docs.cuda(), torch.full((b, S), 40).cuda())
    rule = dict(scale=0.1, cap=cap, slopes=_slopes(n))
    o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
    want = basp.attn_span_bwd(q, k, v, o, lse, do, spans, **rule)
    live = torch.ones(b, S, dtype=torch.bool, device="cuda")
    live[:, 100:133] = False     # the garbage document
    live[1, 250:] = False        # padding
    q2, k2, v2, do2 = (torch.where(live[..., None, None], x, bad) for x in (q, k, v, do))
    o2, lse2 = basp.attn_span_fwd(q2, k2, v2, spans, **rule)
    assert torch.equal(o2[live], o[live])
    assert torch.equal(lse2.transpose(1, 2)[live], lse.transpose(1, 2)[live])
    assert (o2[1, 250:] == 0).all() and (lse2[1, :, 250:] == -math.inf).all()
    assert not o2[:, 100:133].isfinite().any()
    got = basp.attn_span_bwd(q2, k2, v2, o2, lse2, do2, spans, **rule)
    for name, x, y in zip(("dq", "dk", "dv"), got, want):
        assert torch.equal(x[live], y[live]), name
        assert (x[1, 250:] == 0).all(), name


@pytest.mark.parametrize("S", [40, 700])
def test_seen_values_that_are_not_finite(S):
    """A value makes its element NaN in the rows that see it and nothing else."""
    q, k, v, do = _inputs(1, S, 2, 1, 128, seed=13)
    o, _ = basp.attn_span_fwd(q, k, v, None)
    v2 = v.clone()
    v2[0, 10, 0, 5], v2[0, S // 2, 0, 77] = math.inf, math.nan
    o2, _ = basp.attn_span_fwd(q, k, v2, None)
    bad = torch.zeros_like(o, dtype=torch.bool)
    bad[0, 10:, :, 5] = True
    bad[0, S // 2:, :, 77] = True
    assert not o2[bad].isfinite().any()
    assert torch.equal(o2[~bad], o[~bad])


def test_everything_is_padding():
    q, k, v, do = _inputs(2, 200, 4, 2, 96, seed=1)
    spans = torch.zeros(2, 200, 2, dtype=torch.int32, device="cuda")
    o, lse = basp.attn_span_fwd(q, k, v, spans)
    assert (o == 0).all() and (lse == -math.inf).all()
    for x in basp.attn_span_bwd(q, k, v, o, lse, do, spans):
        assert (x == 0).all()


def test_empty():
    for b, S in ((0, 5), (3, 0)):
        q, k, v, do = _inputs(b, S, 4, 2, 64, seed=0)
        o, lse = basp.attn_span_fwd(q, k, v, None)
        assert o.shape == q.shape and lse.shape == (b, 4, S)
        assert [x.shape for x in basp.attn_span_bwd(q, k, v, o, lse, do, None)] == [
            q.shape, k.shape, v.shape]


def test_same_bits_again_and_inside_larger_buffers():
    """Deterministic, and outputs, gradients and the workspace inside larger buffers whose other
    bytes stay as they were; a workspace full of NaN."""
    b, S, n_q, n_k, d = 1, 3100, 8, 2, 128
    q, k, v, do = _inputs(b, S, n_q, n_k, d, seed=21)
    spans = _spans("docs", b, S, 3)
    rule = dict(cap=30.0, slopes=_slopes(n_q))
    o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
    want = basp.attn_span_bwd(q, k, v, o, lse, do, spans, **rule)

    def inside(shape, dtype):
        n = math.prod(shape)
        buf = torch.full((n + 128,), 7.0, device="cuda", dtype=dtype)
        return buf, buf[64:64 + n].view(shape)

    bufs = [inside(q.shape, BF16), inside(lse.shape, F32)]
    basp.attn_span_fwd(q, k, v, spans, out=bufs[0][1], lse=bufs[1][1], **rule)
    assert torch.equal(bufs[0][1], o) and torch.equal(bufs[1][1], lse)
    need = basp.attn_span_bwd_workspace_bytes(b, S, n_q, n_k, d)
    ws = torch.full((need + 512,), 255, device="cuda", dtype=torch.uint8)
    bufs += [inside(x.shape, F32) for x in want]
    for _ in range(2):
        basp.attn_span_bwd(q, k, v, o, lse, do, spans, dq=bufs[2][1], dk=bufs[3][1], dv=bufs[4][1],
                           workspace=ws[256:256 + need], **rule)
        for (buf, x), y in zip(bufs[2:], want):
            assert torch.equal(x, y)
    for buf, x in bufs:
        assert (buf[:64] == 7).all() and (buf[-64:] == 7).all()
    assert (ws[:256] == 255).all() and (ws[-256:] == 255).all()


def test_other_stream_and_graph():
    """On a stream of its own, and captured: replays on new inputs equal eager calls."""
    b, S, n_q, n_k, d = 2, 700, 8, 2, 128
    q, k, v, do = _inputs(b, S, n_q, n_k, d, seed=5)
    spans = _spans("docs", b, S, 3)
    rule = dict(cap=30.0, slopes=_slopes(n_q))
    ws = torch.empty(basp.attn_span_bwd_workspace_bytes(b, S, n_q, n_k, d), device="cuda",
                     dtype=torch.uint8)

    def go():
        o, lse = basp.attn_span_fwd(q, k, v, spans, **rule)
        return o, lse, *basp.attn_span_bwd(q, k, v, o, lse, do, spans, workspace=ws, **rule)

    want = [x.clone() for x in go()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = go()
    side.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go()
    for turn in range(3):
        new = _inputs(b, S, n_q, n_k, d, seed=100 + turn)
        for x, y in zip((q, k, v, do), new):
            x.copy_(y)
        spans.copy_(_spans("wild" if turn == 1 else "prefix", b, S, turn))
        want = [x.clone() for x in go()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, want):
            assert torch.equal(x, y)


def test_attn_spans():
    docs = torch.tensor([[0, 0, 0, 1, 1, -1], [4, 4, 4, 4, 4, 4]], device="cuda")
    pre = torch.tensor([[2, 2, 2, 9, 9, 9], [0, 0, 0, 0, 0, 0]], device="cuda")
    assert basp.attn_spans(docs, pre).tolist() == [
        [[0, 2], [0, 2], [0, 3], [3, 5], [3, 5], [0, 0]], [[0, i + 1] for i in range(6)]]
    assert basp.attn_spans(docs).tolist()[0] == [[0, 1], [0, 2], [0, 3], [3, 4], [3, 5], [0, 0]]


def test_scores_far_apart_in_wide_workgroups():
    """Rows enough for the wider workgroups: P outgrows the reference, within fp32's range and
    past it, and falls below it."""
    q, k, v, do = _inputs(1, 1500, 48, 2, 64, seed=16)
    for span, kind, sign in ((40, "causal", 1), (40, "wild", -1), (250, "docs", 1), (250, "wild", 1),
                             (250, "causal", -1)):
        ramp = torch.linspace(-span, span, 1500, device="cuda")
        k2 = (k.float() * 0.1 + sign * ramp.view(1, -1, 1, 1) / 8).to(BF16)
        q2 = (q.float() * 0.1 + 1).to(BF16)
        spans, slopes = _spans(kind, 1, 1500, 9), None if kind == "docs" else _slopes(48)
        for cap in (None, 60.0):
            print(f"case {span} {kind} {sign} {cap}", flush=True)
            o, lse = basp.attn_span_fwd(q2, k2, v, spans, scale=1.0, cap=cap, slopes=slopes)
            O, bo, L, bl = span_ref.fwd_ref(q2, k2, v, spans, 1.0, cap, slopes)
            check("o", o, O, bo, BF16)
            check("lse", lse, L, bl, F32)


@pytest.mark.parametrize("cap", [None, 30.0, 100.0])
@pytest.mark.parametrize("d", [80, 128])
def test_unseen_values_in_wide_workgroups(cap, d):
    """As test_unseen_values_do_not_count, in the wider workgroups: to the forward's bound, since
    the second pass over such a workgroup adds up in another order."""
    b, S, n = 2, 900, 40
    q, k, v, _ = _inputs(b, S, n, 4, d, seed=12)
    docs = torch.zeros(b, S, dtype=torch.int32)
    docs[:, 300:] = 1
    docs[:, 411:] = 2
    docs[1, 850:] = -1
    spans = basp.attn_spans(docs.cuda(), torch.full((b, S), 100).cuda())
    live = torch.ones(b, S, dtype=torch.bool, device="cuda")
    live[:, 300:411] = False
    live[1, 850:] = False
    slopes = _slopes(n)
    O, bound, L, bl = span_ref.fwd_ref(q, k, v, spans, 0.1, cap, slopes)
    q2, k2, v2 = (torch.where(live[..., None, None], x, math.nan) for x in (q, k, v))
    v2[0, 5, 0, 3] = math.inf     # seen by the first document
    o, lse = basp.attn_span_fwd(q2, k2, v2, spans, scale=0.1, cap=cap, slopes=slopes)
    assert not o[0, :300, :10, 3].isfinite().any()
    o[0, :300, :10, 3] = O[0, :300, :10, 3].to(BF16)
    check("o", o[live], O[live], bound[live], BF16)
    check("lse", lse.transpose(1, 2)[live], L.transpose(1, 2)[live], bl.transpose(1, 2)[live], F32)
    assert (o[1, 850:] == 0).all() and not o[:, 300:411].isfinite().any()
