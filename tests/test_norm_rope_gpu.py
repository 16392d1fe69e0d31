"""Norm and rotation of Q and K, and its backward, against plain fp64."""
import pytest
import torch

import paper_2609_03151_amd as basp
from ops_ref import F64, check, norm_rope_bwd_ref, norm_rope_ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(b, S, n_q, n_k, d, dtype, seed=0, fused=False):
    g = torch.Generator("cuda").manual_seed(seed)
    rn = lambda *s, t=dtype: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    if fused:
        qkv = rn(b, S, n_q + 2 * n_k, d)
        q, k = qkv[:, :, :n_q], qkv[:, :, n_q:n_q + n_k]
    else:
        q, k = rn(b, S, n_q, d), rn(b, S, n_k, d)
    return q, k, 1 + 0.2 * rn(d, t=F32), 1 + 0.2 * rn(d, t=F32), rn


def _run_both(q, k, qw, kw, cos, sin, pos, eps, rot, inter, grad, rn, **more):
    b, S, n_q, d = q.shape
    P = pos if pos is not None else (torch.arange(S, device="cuda")[None] + more.get("pos0", 0)
                                     ).expand(b, S)
    print(f"case {tuple(q.shape)} {tuple(k.shape)} {q.dtype} rot {rot} {inter} {grad}", flush=True)
    qo, ko = basp.qk_norm_rope(q, k, qw, kw, cos, sin, eps=eps, positions=pos, interleaved=inter,
                               **more)
    assert qo.dtype == q.dtype and qo.is_contiguous()
    for name, x, w, y in (("q", q, qw, qo), ("k", k, kw, ko)):
        check(name, y, *norm_rope_ref(x, w, cos, sin, P, eps, rot, inter), x.dtype)
    dqo, dko = rn(*q.shape, t=grad), rn(*k.shape, t=grad)
    dq, dk, dqw, dkw = basp.qk_norm_rope_bwd(q, k, dqo, dko, qw, kw, cos, sin, eps=eps,
                                             positions=pos, interleaved=inter, **more)
    for name, x, dy, w, dx, dw in (("dq", q, dqo, qw, dq, dqw), ("dk", k, dko, kw, dk, dkw)):
        rx, bx, rw, bw = norm_rope_bwd_ref(x, dy, w, cos, sin, P, eps, rot, inter)
        assert dx.dtype == grad
        check(name, dx, rx, bx, grad)
        if w is None:
            assert dw is None
        else:
            check(name + "_weight", dw, rw, bw, F32)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,grad", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_types_and_dims(d, inter, dtype, grad):
    q, k, qw, kw, rn = _inputs(2, 37, 7, 1, d, dtype, seed=d)
    cos, sin = basp.rope_table(64, d)
    _run_both(q, k, qw, kw, cos, sin, None, 1e-6, d, inter, grad, rn)


@pytest.mark.parametrize("b,S,n_q,n_k,d,rot", [
    (1, 1, 1, 1, 128, 128), (1, 1, 8, 1, 64, 32), (3, 1, 8, 2, 128, 64), (1, 1037, 4, 4, 80, 40),
    (5, 13, 28, 4, 96, 48), (2, 512, 4, 4, 64, 64), (1, 300, 3, 3, 128, 8), (1, 31, 2, 1, 80, 0),
])
@pytest.mark.parametrize("inter", [False, True])
def test_sizes_and_partial_rotation(b, S, n_q, n_k, d, rot, inter):
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, BF16, seed=S)
    cos, sin = basp.rope_table(S + 70000, rot) if rot else (None, None)
    _run_both(q, k, qw, kw, cos, sin, None, 1e-5, rot, inter, F32, rn, pos0=69999 if rot else 0)


def test_without_norm_and_strided():
    q, k, _, _, rn = _inputs(2, 29, 7, 1, 96, BF16, fused=True)
    cos, sin = basp.rope_table(29, 96)
    _run_both(q, k, None, None, cos, sin, None, 1e-6, 96, False, F32, rn)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_inputs_and_outputs(dtype):
    """q and k as columns of one projection, outputs as columns of another; the rest untouched."""
    b, S, n_q, n_k, d = 2, 19, 5, 2, 80
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, dtype, fused=True)
    cos, sin = basp.rope_table(S, d)
    want = basp.qk_norm_rope(q.contiguous(), k.contiguous(), qw, kw, cos, sin)
    buf = torch.full((b, S, n_q + n_k + 3, d), 7.0, dtype=dtype, device="cuda")
    basp.qk_norm_rope(q, k, qw, kw, cos, sin, q_out=buf[:, :, 1:1 + n_q],
                      k_out=buf[:, :, 2 + n_q:2 + n_q + n_k])
    assert torch.equal(buf[:, :, 1:1 + n_q], want[0])
    assert torch.equal(buf[:, :, 2 + n_q:2 + n_q + n_k], want[1])
    for c in (0, 1 + n_q, 2 + n_q + n_k):
        assert (buf[:, :, c] == 7).all()
    dy = rn(b, S, n_q, d, t=F32), rn(b, S, n_k, d, t=F32)
    a = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin)
    c = basp.qk_norm_rope_bwd(q.contiguous(), k.contiguous(), *dy, qw, kw, cos, sin)
    assert all(torch.equal(x, y) for x, y in zip(a, c))


def test_in_place():
    q, k, qw, kw, rn = _inputs(2, 77, 8, 2, 128, BF16)
    cos, sin = basp.rope_table(77, 128)
    want = basp.qk_norm_rope(q, k, qw, kw, cos, sin)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    back = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin)
    got = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, dq=dy[0], dk=dy[1])
    assert got[0] is dy[0] and all(torch.equal(x, y) for x, y in zip(got, back))
    basp.qk_norm_rope(q, k, qw, kw, cos, sin, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_padding_and_past_the_table():
    """Given positions in any order; negative ones are padding, ones past the table NaN.  Padding
    may hold anything."""
    b, S, n_q, n_k, d = 3, 41, 4, 2, 128
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, BF16)
    cos, sin = basp.rope_table(500, d)
    pos = torch.randint(0, 500, (b, S), dtype=torch.int32, device="cuda")
    pos[0, 3:9] = -1
    pos[1, 40] = -2 ** 31
    _run_both(q, k, qw, kw, cos, sin, pos, 1e-6, d, False, F32, rn)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    clean = (basp.qk_norm_rope(q, k, qw, kw, cos, sin, positions=pos),
             basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, positions=pos))
    for t in (q, k, *dy):
        t[pos < 0] = torch.nan
    dirty = (basp.qk_norm_rope(q, k, qw, kw, cos, sin, positions=pos),
             basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, positions=pos))
    for c, t in zip(clean, dirty):
        assert all(torch.equal(x, y) for x, y in zip(c, t))
    pos[2, 5], pos[2, 6] = 500, 2 ** 31 - 1
    qo, _ = basp.qk_norm_rope(q, k, qw, kw, cos, sin, positions=pos)
    bad = torch.zeros(b, S, dtype=torch.bool, device="cuda")
    bad[2, 5:7] = True
    assert torch.equal(qo.isnan().all(-1).all(-1), bad) and not qo[~bad].isnan().any()
    dq, _, dqw, _ = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, positions=pos)
    assert dq[bad].isnan().all() and not dq[~bad].isnan().any() and dqw.isnan().all()


def test_extreme_rows():
    """Rows of zeros, of one large value, of the least and the largest magnitudes; a NaN and an
    infinity stay in their own rows."""
    d = 128
    q, k, qw, kw, rn = _inputs(1, 16, 1, 1, d, F32)
    q[0, 0] = 0
    q[0, 1] *= 1e18
    q[0, 2] *= 1e-30
    q[0, 3] = 0
    q[0, 3, 0, 5] = 3.0
    cos, sin = basp.rope_table(16, d)
    _run_both(q, k, qw, kw, cos, sin, None, 1e-6, d, False, F32, rn)
    want, _ = basp.qk_norm_rope(q, k, qw, kw, cos, sin)
    q[0, 7, 0, 3], q[0, 8, 0, 100] = torch.nan, torch.inf
    got, _ = basp.qk_norm_rope(q, k, qw, kw, cos, sin)
    keep = [i for i in range(16) if i not in (7, 8)]
    assert torch.equal(got[0, keep], want[0, keep]) and got[0, 7].isnan().all()


def test_gradient_against_differences():
    """dx and dw against central differences of the forward's own formula in fp64."""
    d, rot, eps, h = 64, 32, 1e-5, 1e-5
    q, k, qw, kw, rn = _inputs(1, 3, 2, 1, d, F32)
    cos, sin = basp.rope_table(3, rot)
    P = torch.arange(3, device="cuda")[None]
    dq_out, dk_out = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    dq, _, dqw, _ = basp.qk_norm_rope_bwd(q, k, dq_out, dk_out, qw, kw, cos, sin, eps=eps)

    def loss(x, w):
        return (norm_rope_ref(x, w, cos, sin, P, eps, rot, False)[0] * dq_out.double()).sum()

    for x, g, f in ((q, dq, lambda t: loss(t, qw)), (qw, dqw, lambda t: loss(q, t))):
        X = x.double()
        for i in range(0, x.numel(), 11):
            e = torch.zeros_like(X)
            e.view(-1)[i] = h
            diff = (f(X + e) - f(X - e)) / (2 * h)
            # differences: h^2 third derivatives, about 1e-10 of values near 1; fp32 sums
            assert abs(diff.item() - g.reshape(-1)[i].item()) < 2e-5, i


@pytest.mark.parametrize("b,S,n_q,n_k,d", [(1, 32768, 8, 2, 128), (4, 4099, 7, 1, 80)])
def test_large_share(b, S, n_q, n_k, d):
    """A whole share: many workgroups and partial sums; twice the same bits."""
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, BF16)
    cos, sin = basp.rope_table(S, d, base=500000.0)
    _run_both(q, k, qw, kw, cos, sin, None, 1e-6, d, False, F32, rn)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    one = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin)
    ws = torch.full((basp.qk_norm_rope_bwd_workspace_bytes(b, S, n_q, n_k, d),), 255,
                    dtype=torch.uint8, device="cuda")
    two = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, workspace=ws)
    assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_shards_before_the_exchange_or_heads_after():
    """The operator commutes with the exchange: all heads of each shard with its pos0, then pack, is
    pack, then the rank's heads, bit for bit."""
    b, S, H, H_kv, d, G, rank = 2, 256, 8, 4, 128, 4, 2
    q, k, qw, kw, _ = _inputs(b, S, H, H_kv, d, BF16)
    cos, sin = basp.rope_table(S, d)
    Sg = S // G
    sh = lambda x: [x[:, j * Sg:(j + 1) * Sg].contiguous() for j in range(G)]  # noqa: E731
    before = [basp.qk_norm_rope(x, y, qw, kw, cos, sin, pos0=j * Sg)
              for j, (x, y) in enumerate(zip(sh(q), sh(k)))]
    qa, ka = basp.pack([x for x, _ in before], rank), basp.pack([y for _, y in before], rank)
    qb, kb = basp.qk_norm_rope(basp.pack(sh(q), rank), basp.pack(sh(k), rank), qw, kw, cos, sin)
    assert torch.equal(qa, qb) and torch.equal(ka, kb)


def test_empty():
    for b, S in ((0, 5), (3, 0)):
        q, k, qw, kw, rn = _inputs(b, S, 4, 2, 64, BF16)
        cos, sin = basp.rope_table(8, 64)
        qo, ko = basp.qk_norm_rope(q, k, qw, kw, cos, sin)
        assert qo.shape == q.shape and ko.shape == k.shape
        _, _, dqw, dkw = basp.qk_norm_rope_bwd(q, k, q.float(), k.float(), qw, kw, cos, sin)
        assert (dqw == 0).all() and (dkw == 0).all()


def test_captured_and_other_stream():
    """Captured once and replayed with new inputs, on a stream of its own, against eager calls."""
    q, k, qw, kw, rn = _inputs(4, 1, 8, 2, 128, BF16)
    cos, sin = basp.rope_table(1000, 128)
    pos = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    ws = torch.empty(basp.qk_norm_rope_bwd_workspace_bytes(4, 1, 8, 2, 128), dtype=torch.uint8,
                     device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    both = lambda w: (*basp.qk_norm_rope(q, k, qw, kw, cos, sin, positions=pos),  # noqa: E731
                      *basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, positions=pos,
                                             workspace=w))
    with torch.cuda.stream(st):
        both(ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            got = both(ws)
    for i in range(4):
        q.copy_(rn(*q.shape))
        dy[0].copy_(rn(*q.shape, t=F32))
        pos.copy_(torch.tensor([[i], [999 - i], [-1], [17 * i]], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = both(None)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i


def test_norm_alone_with_positions():
    """No rotation: positions only mark padding, however large they are."""
    q, k, qw, kw, rn = _inputs(2, 9, 3, 1, 96, BF16)
    pos = torch.arange(18, dtype=torch.int32, device="cuda").view(2, 9) * 10 ** 8
    pos[1, 4] = -3
    qo, ko = basp.qk_norm_rope(q, k, qw, kw, None, None, positions=pos)
    for name, x, w, y in (("q", q, qw, qo), ("k", k, kw, ko)):
        check(name, y, *norm_rope_ref(x, w, None, None, pos, 1e-6, 0, False), BF16)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    dq, dk, dqw, dkw = basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, None, None, positions=pos)
    for name, x, g, w, dx, dw in (("dq", q, dy[0], qw, dq, dqw), ("dk", k, dy[1], kw, dk, dkw)):
        rx, bx, rw, bw = norm_rope_bwd_ref(x, g, w, None, None, pos, 1e-6, 0, False)
        check(name, dx, rx, bx, F32)
        check(name + "_weight", dw, rw, bw, F32)


@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_writes_nothing_else(d):
    """Outputs inside larger buffers: what lies around them stays."""
    b, S, n_q, n_k = 3, 23, 5, 1
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, BF16)
    cos, sin = basp.rope_table(S, d)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)

    def inside(n, dtype, shape):
        buf = torch.full((n + 128,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[64:64 + n].view(shape)

    outs = {n: inside(t.numel(), dt, t.shape) for n, t, dt in (
        ("q_out", q, BF16), ("k_out", k, BF16), ("dq", q, F32), ("dk", k, F32),
        ("dq_weight", qw, F32), ("dk_weight", kw, F32))}
    ws, space = inside(basp.qk_norm_rope_bwd_workspace_bytes(b, S, n_q, n_k, d) // 4, F32, (-1,))
    view = lambda *names: {n: outs[n][1] for n in names}  # noqa: E731
    basp.qk_norm_rope(q, k, qw, kw, cos, sin, **view("q_out", "k_out"))
    basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, cos, sin, workspace=space,
                          **view("dq", "dk", "dq_weight", "dk_weight"))
    for buf in [ws, *(x[0] for x in outs.values())]:
        assert (buf[:64] == 7).all() and (buf[-64:] == 7).all()
    want = basp.qk_norm_rope(q, k, qw, kw, cos, sin)
    assert torch.equal(outs["q_out"][1], want[0]) and torch.equal(outs["k_out"][1], want[1])


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_reads_its_rows_alone(d, dtype):
    """NaN around the heads that a call takes, in rows shorter than their lanes and head counts that
    leave a group short, reaches neither outputs nor gradients."""
    b, S, n_q, n_k = 2, 21, 5, 2
    q, k, qw, kw, rn = _inputs(b, S, n_q, n_k, d, dtype, seed=d)
    cos, sin = basp.rope_table(S, d)
    buf = torch.full((b, S, n_q + n_k + 3, d), torch.nan, dtype=dtype, device="cuda")
    buf[:, :, 1:1 + n_q], buf[:, :, 2 + n_q:2 + n_q + n_k] = q, k
    _run_both(buf[:, :, 1:1 + n_q], buf[:, :, 2 + n_q:2 + n_q + n_k], qw, kw, cos, sin, None, 1e-6,
              d, False, F32, rn)


def test_norm_alone_behind_any_position():
    """No rotation: pos0 has no effect, however large."""
    q, k, qw, kw, rn = _inputs(2, 9, 3, 1, 80, BF16)
    dy = rn(*q.shape, t=F32), rn(*k.shape, t=F32)
    both = [(*basp.qk_norm_rope(q, k, qw, kw, None, None, pos0=p),
             *basp.qk_norm_rope_bwd(q, k, *dy, qw, kw, None, None, pos0=p)) for p in (0, 2 ** 31 - 1)]
    assert all(torch.equal(x, y) for x, y in zip(*both)) and both[0][0].any()
