"""Python binding of libbasp: one GPU's share of batch-aware Ulysses attention.

Argument marshalling only: every function checks tensor devices, dtypes and
contiguity, then passes raw device pointers, sizes and the current HIP stream
to the C ABI of ``include/basp.h``.  All work runs in the library's HIP
kernels; there is no fallback.  If ``libbasp.so`` has not been built, importing
the library raises.

Names follow the C ABI: ``pack``, ``unpack``, ``attn_fwd``, ``attn_bwd``,
``attn_bwd_workspace_bytes``, ``qk_norm_rope``, ``kv_write``, ``attn_decode``,
``validate``, ``group_of``, ``status_str``.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbasp.so")

BASP_BF16, BASP_F32, BASP_E4M3 = 0, 1, 2
STATUS = {
    0: "BASP_OK", 1: "BASP_ERR_NULL", 2: "BASP_ERR_SHAPE", 3: "BASP_ERR_RANK",
    4: "BASP_ERR_UNSUPPORTED", 5: "BASP_ERR_ALIGN", 6: "BASP_ERR_WORKSPACE",
    7: "BASP_ERR_HIP", 8: "BASP_ERR_DP_FALLBACK",
}
# Every symbol include/basp.h declares.
EXPORTS = ("basp_status_str", "basp_group_of", "basp_validate", "basp_pack",
           "basp_unpack", "basp_unpack_add", "basp_pack_qkv", "basp_unpack_pack",
           "basp_unpack_grads", "basp_a2a_pack", "basp_a2a_unpack",
           "basp_a2a_pack_bf16", "basp_attn_fwd",
           "basp_attn_fwd_sharded", "basp_attn_bwd_workspace_bytes", "basp_attn_bwd",
           "basp_attn_bwd_noalloc", "basp_attn_bwd_sharded_workspace_bytes",
           "basp_attn_bwd_sharded",
           "basp_qk_norm_rope", "basp_qk_norm_rope_bwd",
           "basp_qk_norm_rope_bwd_workspace_bytes", "basp_kv_write", "basp_kv_read",
           "basp_attn_decode", "basp_attn_decode_workspace_bytes")
# Bytes of the static device buffer basp_attn_bwd_noalloc works in.
NOALLOC_SCRATCH_BYTES = 128 << 20


class BaspError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_str(status)}")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libbasp.so; raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
            "or `python paper_2609_03151_amd/build.py`")
    L = ctypes.CDLL(LIB_PATH)
    i, vp, sz, f = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    ip = ctypes.POINTER(ctypes.c_int)
    L.basp_status_str.argtypes = [i]
    L.basp_status_str.restype = ctypes.c_char_p
    L.basp_group_of.argtypes = [i, i, i, ip, ip, ip]
    L.basp_validate.argtypes = [i] * 7
    L.basp_pack.argtypes = [ctypes.POINTER(vp), vp] + [i] * 7 + [vp]
    L.basp_unpack.argtypes = [vp, ctypes.POINTER(vp)] + [i] * 7 + [vp]
    L.basp_unpack_add.argtypes = [vp, ctypes.POINTER(vp)] + [i] * 6 + [vp]
    L.basp_pack_qkv.argtypes = [ctypes.POINTER(vp)] * 3 + [vp] * 3 + [i] * 8 + [vp]
    L.basp_unpack_pack.argtypes = [vp] + [ctypes.POINTER(vp)] * 2 + [vp] + [i] * 7 + [vp]
    L.basp_unpack_grads.argtypes = [vp] * 3 + [ctypes.POINTER(vp)] * 3 + [i] * 7 + [vp]
    L.basp_a2a_pack.argtypes = [vp, vp] + [i] * 6 + [vp]
    L.basp_a2a_unpack.argtypes = [vp, vp] + [i] * 6 + [vp]
    L.basp_a2a_pack_bf16.argtypes = [vp, vp] + [i] * 5 + [vp]
    L.basp_attn_fwd.argtypes = [vp] * 5 + [i] * 6 + [f, vp]
    L.basp_attn_bwd_workspace_bytes.argtypes = [i] * 6
    L.basp_attn_bwd_workspace_bytes.restype = sz
    L.basp_attn_bwd_sharded_workspace_bytes.argtypes = [i] * 6
    L.basp_attn_bwd_sharded_workspace_bytes.restype = sz
    L.basp_attn_bwd.argtypes = [vp] * 10 + [sz] + [i] * 6 + [f, vp]
    L.basp_attn_bwd_noalloc.argtypes = [vp] * 9 + [i] * 6 + [f, vp]
    tab = ctypes.POINTER(vp)
    L.basp_attn_fwd_sharded.argtypes = [tab] * 4 + [vp] + [i] * 7 + [f, vp]
    L.basp_attn_bwd_sharded.argtypes = ([tab] * 4 + [vp] + [tab] * 4 + [vp, sz] + [i] * 7
                                        + [f, vp])
    ll = ctypes.c_longlong
    L.basp_qk_norm_rope.argtypes = [vp] * 9 + [i] * 7 + [ll] * 4 + [f] + [i] * 3 + [vp]
    L.basp_qk_norm_rope_bwd_workspace_bytes.argtypes = [i] * 5
    L.basp_qk_norm_rope_bwd_workspace_bytes.restype = sz
    L.basp_qk_norm_rope_bwd.argtypes = ([vp] * 14 + [sz] + [i] * 7 + [ll] * 2 + [f] + [i] * 4
                                        + [vp])
    L.basp_kv_write.argtypes = [vp] * 9 + [i] * 7 + [ll] * 2 + [i, vp]
    L.basp_kv_read.argtypes = [vp] * 9 + [i] * 8 + [vp]
    L.basp_attn_decode_workspace_bytes.argtypes = [i] * 5
    L.basp_attn_decode_workspace_bytes.restype = sz
    L.basp_attn_decode.argtypes = [vp] * 10 + [sz] + [i] * 8 + [ll, f, i, vp]
    for name in ("basp_group_of", "basp_validate", "basp_pack", "basp_unpack",
                 "basp_a2a_pack", "basp_a2a_unpack", "basp_a2a_pack_bf16", "basp_attn_fwd",
                 "basp_attn_bwd",
                 "basp_attn_bwd_noalloc"):
        getattr(L, name).restype = i
    _lib = L
    return L


def status_str(status: int) -> str:
    return lib().basp_status_str(int(status)).decode()


def _check(rc: int, what: str):
    if rc != 0:
        raise BaspError(rc, what)


# A small share's calls take about as long on the host as on the GPU, so the
# marshalling below avoids temporary objects: raw integers for pointers and for
# the stream (torch's raw stream handle, 0.1 us, instead of a Stream object, 2
# us), one array type per table length.
def _stream(t: torch.Tensor) -> int:
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _dev(t: torch.Tensor, name: str, dtype=None) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


_table_types: dict = {}


def _table(tensors, name: str, dtype, n: int):
    """Pointer table of n device tensors, each checked as _dev does (missing ones are NULL)."""
    kind = _table_types.get(n)
    if kind is None:
        kind = _table_types[n] = ctypes.c_void_p * n
    ptrs = []
    for t in tensors:  # once: the caller may pass an iterator
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()
                and t.dtype == dtype):
            _dev(t, f"{name}[{len(ptrs)}]", dtype)  # raises: says which tensor, and why
        ptrs.append(t.data_ptr())
    return kind(*ptrs)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BASP_BF16
    if t.dtype == torch.float32:
        return BASP_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


# ------------------------------------------------------------ host helpers
def group_of(world: int, micro_batch: int, global_rank: int):
    """(group, local_rank, group_size) of a global rank (Alg. 1 / Alg. 2)."""
    g, l, k = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib().basp_group_of(world, micro_batch, global_rank, ctypes.byref(g),
                               ctypes.byref(l), ctypes.byref(k)), "basp_group_of")
    return g.value, l.value, k.value


def validate(b, S, H, H_kv, d, G, rank) -> int:
    """Status code of a share's parameters (0 = valid); no GPU needed."""
    return lib().basp_validate(b, S, H, H_kv, d, G, rank)


# ------------------------------------------------------------ permutations
def heads_per_member(n: int, G: int) -> int:
    """Heads of an n-head tensor one member handles: n/G, or 1 for a head
    shared by G/n members (n < G, G divisible by n); 0 if neither holds."""
    if n % G == 0:
        return n // G
    return 1 if (n < G and G % n == 0) else 0


def pack(shards, rank: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """G shards [b, S/G, n, d] -> the rank's head-sharded [b, S, nl, d]."""
    G = len(shards)
    b, Sg, n, d = shards[0].shape
    ptrs = _table(shards, "shards", shards[0].dtype, G)
    shape, device = shards[0].shape, shards[0].device
    for s in shards:
        if s.shape != shape or s.device != device:
            raise ValueError("shards differ in shape or device")
    if out is None:
        out = torch.empty((b, Sg * G, heads_per_member(n, G), d), dtype=shards[0].dtype,
                          device=shards[0].device)
    _check(lib().basp_pack(ptrs, _dev(out, "out", shards[0].dtype), b, Sg * G, n, d, G, rank,
                           _dtype_code(out), _stream(out)), "basp_pack")
    return out


def unpack(local: torch.Tensor, shards, rank: int):
    """Write local [b, S, n/G, d] into the rank's head slice of every shard."""
    G = len(shards)
    b, Sg, n, d = shards[0].shape
    ptrs = _table(shards, "shards", local.dtype, G)
    _check(lib().basp_unpack(_dev(local, "local"), ptrs, b, Sg * G, n, d, G, rank,
                             _dtype_code(local), _stream(local)), "basp_unpack")
    return shards


def unpack_add(local: torch.Tensor, shards, rank: int):
    """fp32: add local [b, S, nl, d] into the rank's head slice of every shard
    (gradients of kv heads that several members share)."""
    G = len(shards)
    b, Sg, n, d = shards[0].shape
    ptrs = _table(shards, "shards", torch.float32, G)
    _check(lib().basp_unpack_add(_dev(local, "local", torch.float32), ptrs, b, Sg * G, n, d, G,
                                 rank, _stream(local)), "basp_unpack_add")
    return shards


def pack_qkv(q_shards, k_shards, v_shards, rank: int, q=None, k=None, v=None):
    """pack of Q, K and V in one call (one launch when G <= 16); returns (q, k, v)."""
    G = len(q_shards)
    b, Sg, H, d = q_shards[0].shape
    H_kv = k_shards[0].shape[2]
    dt = q_shards[0].dtype
    dev = q_shards[0].device
    if q is None:
        q = torch.empty((b, Sg * G, heads_per_member(H, G), d), dtype=dt, device=dev)
    if k is None:
        k = torch.empty((b, Sg * G, heads_per_member(H_kv, G), d), dtype=dt, device=dev)
    if v is None:
        v = torch.empty_like(k)
    _check(lib().basp_pack_qkv(_table(q_shards, "q_shards", dt, G),
                               _table(k_shards, "k_shards", dt, G),
                               _table(v_shards, "v_shards", dt, G), _dev(q, "q", dt),
                               _dev(k, "k", dt),
                               _dev(v, "v", dt), b, Sg * G, H, H_kv, d, G, rank, _dtype_code(q),
                               _stream(q)), "basp_pack_qkv")
    return q, k, v


def unpack_pack(local: torch.Tensor, shards, src_shards, rank: int, out: torch.Tensor):
    """unpack of ``local`` into ``shards``, then pack of ``src_shards`` into ``out``, in one call
    (one launch when G <= 16); all of one dtype and head count, and no buffer of one in the other."""
    G = len(shards)
    b, Sg, n, d = shards[0].shape
    dt = local.dtype
    if len(src_shards) != G:
        raise ValueError("src_shards and shards differ in number")
    src = _table(src_shards, "src_shards", dt, G)
    shape, device = shards[0].shape, local.device
    for t in src_shards:
        if t.shape != shape or t.device != device:
            raise ValueError("shards differ in shape or device")
    _check(lib().basp_unpack_pack(_dev(local, "local"), _table(shards, "shards", dt, G), src,
                                  _dev(out, "out", dt), b, Sg * G, n, d, G, rank,
                                  _dtype_code(local), _stream(local)), "basp_unpack_pack")
    return out


def unpack_grads(dq, dk, dv, dq_shards, dk_shards, dv_shards, rank: int):
    """fp32 unpack of dQ, dK, dV in one call; dK, dV are added into the shards
    when the rank's kv head is shared (H_kv < G)."""
    G = len(dq_shards)
    b, Sg, H, d = dq_shards[0].shape
    H_kv = dk_shards[0].shape[2]
    f32 = torch.float32
    _check(lib().basp_unpack_grads(_dev(dq, "dq", f32), _dev(dk, "dk", f32), _dev(dv, "dv", f32),
                                   _table(dq_shards, "dq_shards", f32, G),
                                   _table(dk_shards, "dk_shards", f32, G),
                                   _table(dv_shards, "dv_shards", f32, G), b, Sg * G, H, H_kv, d,
                                   G, rank, _stream(dq)), "basp_unpack_grads")


def a2a_pack(own: torch.Tensor, G: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """Own shard [b, S/G, n, d] -> send buffer [G, b, S/G, nl, d], one block per member."""
    b, Sg, n, d = own.shape
    if out is None:
        out = torch.empty((G, b, Sg, heads_per_member(n, G), d), dtype=own.dtype,
                          device=own.device)
    _check(lib().basp_a2a_pack(_dev(own, "own"), _dev(out, "out", own.dtype), b, Sg * G, n, d,
                               G, _dtype_code(own), _stream(own)), "basp_a2a_pack")
    return out


def a2a_pack_bf16(own: torch.Tensor, G: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """fp32 own shard [b, S/G, n, d] -> bf16 send buffer [G, b, S/G, nl, d]
    (a2a_pack with the conversion to bf16, round to nearest even, fused)."""
    b, Sg, n, d = own.shape
    if out is None:
        out = torch.empty((G, b, Sg, heads_per_member(n, G), d), dtype=torch.bfloat16,
                          device=own.device)
    _check(lib().basp_a2a_pack_bf16(_dev(own, "own", torch.float32),
                                    _dev(out, "out", torch.bfloat16), b, Sg * G, n, d, G,
                                    _stream(own)), "basp_a2a_pack_bf16")
    return out


def a2a_unpack(recv: torch.Tensor, out: torch.Tensor | None = None,
               n_heads: int | None = None) -> torch.Tensor:
    """Received blocks [G, b, S/G, n/G, d] -> own shard [b, S/G, n, d].

    ``n_heads`` < G: fp32 gradients of shared heads, blocks [G, b, S/G, 1, d]
    summed per head in member order."""
    G, b, Sg, nl, d = recv.shape
    n = G * nl if n_heads is None else n_heads
    if out is None:
        out = torch.empty((b, Sg, n, d), dtype=recv.dtype, device=recv.device)
    _check(lib().basp_a2a_unpack(_dev(recv, "recv"), _dev(out, "out", recv.dtype), b, Sg * G,
                                 n, d, G, _dtype_code(recv), _stream(recv)),
           "basp_a2a_unpack")
    return out


# -------------------------------------------------------------- attention
def _attn_dims(q, k, G, H_kv):
    b, S, Hl, d = q.shape
    Hkl = k.shape[2]
    if k.shape[:2] != (b, S) or k.shape[3] != d:
        raise ValueError("q and k/v disagree in shape")
    if H_kv is None:
        H_kv = Hkl * G
    elif heads_per_member(H_kv, G) != Hkl:
        raise ValueError(f"k/v hold {Hkl} heads; a member of {G} handles "
                         f"{heads_per_member(H_kv, G)} of {H_kv}")
    return b, S, Hl * G, H_kv, d


def attn_fwd(q, k, v, G: int = 1, scale: float | None = None, out=None, lse=None,
             H_kv: int | None = None):
    """Causal GQA attention of the local heads: returns (o bf16, lse fp32 [b,Hl,S]).

    ``H_kv``: global kv heads (default: k's heads times G); give it when fewer
    kv heads than members share one head per member."""
    b, S, H, H_kv, d = _attn_dims(q, k, G, H_kv)
    scale = d ** -0.5 if scale is None else scale
    if v.shape != k.shape:
        raise ValueError("v must have k's shape")
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((b, q.shape[2], S), dtype=torch.float32, device=q.device)
    _check(lib().basp_attn_fwd(_dev(q, "q", torch.bfloat16), _dev(k, "k", torch.bfloat16),
                               _dev(v, "v", torch.bfloat16), _dev(out, "o", torch.bfloat16),
                               _dev(lse, "lse", torch.float32), b, S, H, H_kv, d, G,
                               float(scale), _stream(q)), "basp_attn_fwd")
    return out, lse


def attn_bwd_workspace_bytes(b, S, H, H_kv, d, G) -> int:
    return int(lib().basp_attn_bwd_workspace_bytes(b, S, H, H_kv, d, G))


def attn_bwd_sharded_workspace_bytes(b, S, H, H_kv, d, G) -> int:
    return int(lib().basp_attn_bwd_sharded_workspace_bytes(b, S, H, H_kv, d, G))


def attn_bwd(q, k, v, o, lse, do, G: int = 1, scale: float | None = None,
             dq=None, dk=None, dv=None, workspace=None, H_kv: int | None = None):
    """Backward of attn_fwd: returns (dq, dk, dv) in fp32."""
    b, S, H, H_kv, d = _attn_dims(q, k, G, H_kv)
    scale = d ** -0.5 if scale is None else scale
    if dq is None:
        dq = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=torch.float32, device=q.device)
    if dv is None:
        dv = torch.empty(v.shape, dtype=torch.float32, device=q.device)
    if workspace is None:
        need = attn_bwd_workspace_bytes(b, S, H, H_kv, d, G)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _check(lib().basp_attn_bwd(
        _dev(q, "q", torch.bfloat16), _dev(k, "k", torch.bfloat16),
        _dev(v, "v", torch.bfloat16), _dev(o, "o", torch.bfloat16),
        _dev(lse, "lse", torch.float32), _dev(do, "do", torch.bfloat16),
        _dev(dq, "dq", torch.float32), _dev(dk, "dk", torch.float32),
        _dev(dv, "dv", torch.float32), _dev(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), b, S, H, H_kv, d, G, float(scale),
        _stream(q)), "basp_attn_bwd")
    return dq, dk, dv


def attn_bwd_noalloc(q, k, v, o, lse, do, dq, dk, dv, G: int = 1, scale: float | None = None,
                     H_kv: int | None = None):
    """attn_bwd into caller-given dq, dk, dv (fp32) with no workspace argument:
    the library's static device buffer serves instead (basp_attn_bwd_noalloc)."""
    b, S, H, H_kv, d = _attn_dims(q, k, G, H_kv)
    scale = d ** -0.5 if scale is None else scale
    _check(lib().basp_attn_bwd_noalloc(
        _dev(q, "q", torch.bfloat16), _dev(k, "k", torch.bfloat16),
        _dev(v, "v", torch.bfloat16), _dev(o, "o", torch.bfloat16),
        _dev(lse, "lse", torch.float32), _dev(do, "do", torch.bfloat16),
        _dev(dq, "dq", torch.float32), _dev(dk, "dk", torch.float32),
        _dev(dv, "dv", torch.float32), b, S, H, H_kv, d, G, float(scale),
        _stream(q)), "basp_attn_bwd_noalloc")
    return dq, dk, dv


# ------------------------------------------------- attention on the shards
def _shards(shards, name: str, dtype, G: int):
    return _table(shards, name, dtype, max(G, len(shards)))


def attn_fwd_sharded(q_shards, k_shards, v_shards, o_shards, rank: int,
                     scale: float | None = None, lse=None):
    """Attention of the rank's heads read from the G sequence shards (each
    [b, S/G, H or H_kv, d] bf16) and written into the rank's head slice of
    o_shards; returns lse [b, H/G, S]."""
    G = len(q_shards)
    b, Sg, H, d = q_shards[0].shape
    H_kv = k_shards[0].shape[2]
    S = Sg * G
    scale = d ** -0.5 if scale is None else scale
    if lse is None:
        lse = torch.empty((b, H // G, S), dtype=torch.float32, device=q_shards[0].device)
    bf = torch.bfloat16
    _check(lib().basp_attn_fwd_sharded(
        _shards(q_shards, "q", bf, G), _shards(k_shards, "k", bf, G), _shards(v_shards, "v", bf, G),
        _shards(o_shards, "o", bf, G), _dev(lse, "lse", torch.float32), b, S, H, H_kv, d, G, rank,
        float(scale), _stream(lse)), "basp_attn_fwd_sharded")
    return lse


def attn_bwd_sharded(q_shards, k_shards, v_shards, o_shards, lse, do_shards, dq_shards,
                     dk_shards, dv_shards, rank: int, scale: float | None = None,
                     workspace=None):
    """Backward of attn_fwd_sharded: dQ, dK, dV (fp32) into the rank's head
    slices of their shard buffers.  With a shared kv head (H_kv < G),
    dk_shards / dv_shards are the G send blocks [b, S/G, 1, d] of this
    member's partial dK, dV instead."""
    G = len(q_shards)
    b, Sg, H, d = q_shards[0].shape
    H_kv = k_shards[0].shape[2]
    S = Sg * G
    scale = d ** -0.5 if scale is None else scale
    if workspace is None:
        need = attn_bwd_sharded_workspace_bytes(b, S, H, H_kv, d, G)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=lse.device)
    bf, f32 = torch.bfloat16, torch.float32
    _check(lib().basp_attn_bwd_sharded(
        _shards(q_shards, "q", bf, G), _shards(k_shards, "k", bf, G), _shards(v_shards, "v", bf, G),
        _shards(o_shards, "o", bf, G), _dev(lse, "lse", f32), _shards(do_shards, "do", bf, G),
        _shards(dq_shards, "dq", f32, G), _shards(dk_shards, "dk", f32, G),
        _shards(dv_shards, "dv", f32, G),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
        b, S, H, H_kv, d, G, rank, float(scale), _stream(lse)), "basp_attn_bwd_sharded")


# --------------------------------------- operators around attention
# A call on a few tokens takes less time on the GPU than its arguments' checks
# would as so many Python calls: one condition per tensor below, and a refusal's
# wording found only once it is refused.  All tensors of a call lie on one
# device, which is made current for the launch if it is not.
_Tensor, _F32, _BF, _I32 = torch.Tensor, torch.float32, torch.bfloat16, torch.int32


def _call(name: str, fn, dev: int, *args):
    if dev < 0:
        raise TypeError(f"{name}: tensors must be CUDA (HIP) tensors")
    if dev == torch._C._cuda_getDevice():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if rc != 0:
        raise BaspError(rc, name)


def _int(x: int) -> int:
    """A size as a C int: -1, which the library refuses, for one that does not fit."""
    return x if -1 < x < 1 << 31 else -1


def _device(t, name: str, dims: int) -> int:
    """Device index of a call's first tensor, of this many dimensions; below zero for a host tensor,
    which _call refuses."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions, got {t.dim()}")
    return t.get_device()


def _refuse(t, name: str, dtype, shape, dev: int):
    if dev >= 0 or not isinstance(t, _Tensor):
        _dev(t, name, dtype)
    elif t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} is on device {t.get_device()}, the call's first tensor on {dev}")


def _on(t, name: str, dtype, shape, dev: int) -> int:
    """Pointer of a contiguous tensor of this type and shape on device ``dev``."""
    if (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        return t.data_ptr()
    _refuse(t, name, dtype, shape, dev)


def _two(a, a_name: str, b, b_name: str, dtype, shape, dev: int):
    """Pointers of two such tensors."""
    if (isinstance(a, _Tensor) and isinstance(b, _Tensor) and a.dtype is dtype and b.dtype is dtype
            and a.shape == shape == b.shape and a.get_device() == dev == b.get_device()
            and a.is_contiguous() and b.is_contiguous()):
        return a.data_ptr(), b.data_ptr()
    return _on(a, a_name, dtype, shape, dev), _on(b, b_name, dtype, shape, dev)


def _rows(t, name: str, dtype, shape, dev: int):
    """(pointer, elements between tokens) of a [..., n, d] tensor whose tokens lie one stride apart
    and whose heads lie side by side: contiguous, or columns of a wider contiguous tensor."""
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape
            and t.get_device() == dev):
        _refuse(t.contiguous() if isinstance(t, _Tensor) else t, name, dtype, shape, dev)
    n, d = shape[-2], shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), n * d
    st = t.stride()
    lead = [(s, z) for s, z in zip(st[:-2], shape[:-2]) if z > 1]  # outermost first
    row = lead[-1][0] if lead else n * d
    ok = st[-1] == 1 and (n == 1 or st[-2] == d) and row >= n * d
    want = row
    for s, z in reversed(lead):
        ok = ok and s == want
        want = s * z
    if not ok:
        raise ValueError(f"{name} must have its heads side by side and its tokens one stride apart")
    return t.data_ptr(), row


def _like(t):
    """A new contiguous tensor of t's shape and type (empty_like keeps the order of dimensions
    otherwise, and asking for another costs half a microsecond)."""
    if t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _space(workspace, need: int, like, dev: int):
    """(tensor to keep, pointer, bytes) of a given workspace of any type, or of a new one."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = like.new_empty(need, dtype=torch.uint8)
        return workspace, workspace.data_ptr(), need
    p = _on(workspace, "workspace", workspace.dtype, workspace.shape, dev)
    return workspace, p, workspace.numel() * workspace.element_size()


def _norm_args(q, k, q_weight, k_weight, cos, sin, positions):
    """Device, sizes, (weights, tables, positions) pointers and the element type's code."""
    dev = _device(q, "q", 4)
    b, S, n_q, d = q.shape
    if not isinstance(k, _Tensor) or k.dim() != 4:
        raise ValueError("k must be [b, S, n_k, d]")
    kb, kS, n_k, kd = k.shape
    if kb != b or kS != S or kd != d:
        raise ValueError("q and k disagree in shape")
    if (cos is None) != (sin is None) or (q_weight is None) != (k_weight is None):
        raise ValueError("cos and sin, and q_weight and k_weight, go together")
    qw = kw = c = sn = None
    if q_weight is not None:
        qw, kw = _two(q_weight, "q_weight", k_weight, "k_weight", _F32, (d,), dev)
    rows = half = 0
    if cos is not None:
        if not isinstance(cos, _Tensor) or cos.dim() != 2:
            raise ValueError("cos and sin must be [positions, rot/2]")
        table = cos.shape
        rows, half = table
        c, sn = _two(cos, "cos", sin, "sin", _F32, table, dev)
        if half == 0:  # no columns: nothing is rotated
            c = sn = None
    pos = None if positions is None else _on(positions, "positions", _I32, (b, S), dev)
    return dev, (b, S, n_q, n_k, d, 2 * half, _int(rows)), (qw, kw), (c, sn, pos), _dtype_code(q)


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, eps: float = 1e-6, positions=None,
                 pos0: int = 0, interleaved: bool = False, q_out=None, k_out=None):
    """RMS norm of every query and key head, and the position rotation, in one pass.

    ``q`` [b, S, n_q, d], ``k`` [b, S, n_k, d] bf16 or fp32 (columns of a fused projection's output
    will do); weights fp32 [d], or both None for no norm; ``cos``, ``sin`` fp32 [positions, rot/2]
    (``rope_table`` makes them), or both None for no rotation.  A token's position is
    ``positions`` int32 [b, S] (negative: a row of padding, zeros out), or pos0 + its index.
    Returns (q_out, k_out) in q's type; ``q_out`` may be ``q`` itself, ``k_out`` ``k``."""
    dev, dims, w, turn, code = _norm_args(q, k, q_weight, k_weight, cos, sin, positions)
    dt, q_shape, k_shape, d = q.dtype, q.shape, k.shape, dims[4]
    qp, q_row = _rows(q, "q", dt, q_shape, dev)
    kp, k_row = _rows(k, "k", dt, k_shape, dev)
    if q_out is None:
        q_out = _like(q)
        qop, qo_row = q_out.data_ptr(), dims[2] * d
    else:
        qop, qo_row = _rows(q_out, "q_out", dt, q_shape, dev)
    if k_out is None:
        k_out = _like(k)
        kop, ko_row = k_out.data_ptr(), dims[3] * d
    else:
        kop, ko_row = _rows(k_out, "k_out", dt, k_shape, dev)
    _call("basp_qk_norm_rope", (_lib or lib()).basp_qk_norm_rope, dev, qp, kp, qop, kop, *w, *turn,
          *dims, q_row, k_row, qo_row, ko_row, eps, _int(pos0), interleaved, code)
    return q_out, k_out


def qk_norm_rope_bwd_workspace_bytes(b, S, n_q, n_k, d) -> int:
    return int(lib().basp_qk_norm_rope_bwd_workspace_bytes(b, S, n_q, n_k, d))


def qk_norm_rope_bwd(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, eps: float = 1e-6,
                     positions=None, pos0: int = 0, interleaved: bool = False, dq=None, dk=None,
                     dq_weight=None, dk_weight=None, workspace=None):
    """Backward of qk_norm_rope at its inputs ``q``, ``k``: from the gradients of its outputs (fp32
    or bf16, contiguous) to (dq, dk, dq_weight, dk_weight): dq, dk in the gradients' type (``dq``
    may be ``dq_out`` itself, ``dk`` ``dk_out``), the weights' in fp32 (None without weights)."""
    dev, dims, w, turn, code = _norm_args(q, k, q_weight, k_weight, cos, sin, positions)
    b, S, n_q, n_k, d = dims[:5]
    q_shape, k_shape = q.shape, k.shape
    qp, q_row = _rows(q, "q", q.dtype, q_shape, dev)
    kp, k_row = _rows(k, "k", q.dtype, k_shape, dev)
    if not isinstance(dq_out, _Tensor):
        raise TypeError("dq_out must be a CUDA (HIP) tensor")
    gt, gcode = dq_out.dtype, _dtype_code(dq_out)
    gq, gk = _on(dq_out, "dq_out", gt, q_shape, dev), _on(dk_out, "dk_out", gt, k_shape, dev)
    if dq is None:
        dq = torch.empty_like(dq_out)
        dqp = dq.data_ptr()
    else:
        dqp = _on(dq, "dq", gt, q_shape, dev)
    if dk is None:
        dk = torch.empty_like(dk_out)
        dkp = dk.data_ptr()
    else:
        dkp = _on(dk, "dk", gt, k_shape, dev)
    L = _lib or lib()
    dqw = dkw = ws = ws_n = None
    if q_weight is None:
        dq_weight = dk_weight = None
        ws_n = 0
    else:
        if dq_weight is None:
            dq_weight = torch.empty_like(q_weight)
            dqw = dq_weight.data_ptr()
        else:
            dqw = _on(dq_weight, "dq_weight", _F32, (d,), dev)
        if dk_weight is None:
            dk_weight = torch.empty_like(k_weight)
            dkw = dk_weight.data_ptr()
        else:
            dkw = _on(dk_weight, "dk_weight", _F32, (d,), dev)
        if b * S == 0:
            dq_weight.zero_()
            dk_weight.zero_()
        need = 0 if workspace is not None else L.basp_qk_norm_rope_bwd_workspace_bytes(
            b, S, n_q, n_k, d)
        workspace, ws, ws_n = _space(workspace, need, q, dev)
    _call("basp_qk_norm_rope_bwd", L.basp_qk_norm_rope_bwd, dev, qp, kp, gq, gk, dqp, dkp, *w, dqw,
          dkw, *turn, ws, ws_n, *dims, q_row, k_row, eps, _int(pos0), interleaved, code, gcode)
    return dq, dk, dq_weight, dk_weight


def rope_table(n: int, rot: int, base: float = 10000.0, device="cuda"):
    """cos, sin fp32 [n, rot/2] of positions 0 .. n-1, angle p * base^(-2i/rot), formed in 64 bits
    (an fp32 angle is off by 2^-8 at a position of 128K)."""
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(n, dtype=torch.float64, device=device)[:, None] * freq
    return ang.cos().float(), ang.sin().float()


# --------------------------------------------------------- key-value cache
_CACHE_TYPES = {torch.bfloat16: BASP_BF16, torch.float8_e4m3fn: BASP_E4M3}


def _pages(k_pages, v_pages, k_scales, v_scales, table, b, dev: int):
    """((k_pages, v_pages, k_scales, v_scales, table) pointers, (n_k, d, page, n_pages, max_pages),
    dtype code) of a paged cache whose table has b rows."""
    if not isinstance(k_pages, _Tensor) or k_pages.dim() != 4:
        raise ValueError("k_pages must be [n_pages, n_k, page, d]")
    shape = k_pages.shape
    n_pages, n_k, page, d = shape
    dt = k_pages.dtype
    code = _CACHE_TYPES.get(dt)
    if code is None:
        raise TypeError(f"unsupported dtype {dt}")
    if not isinstance(table, _Tensor) or table.dim() != 2 or table.shape[0] != b:
        raise ValueError(f"block_table must be [{b}, max_pages]")
    if code == BASP_BF16:
        if k_scales is not None or v_scales is not None:
            raise ValueError("a bf16 cache has no scales")
        ks = vs = None
    else:
        if k_scales is None or v_scales is None:
            raise ValueError("an 8-bit cache has k_scales and v_scales")
        ks, vs = _two(k_scales, "k_scales", v_scales, "v_scales", torch.uint8, (n_pages, n_k, page),
                      dev)
    t_shape = table.shape
    return ((*_two(k_pages, "k_pages", v_pages, "v_pages", dt, shape, dev), ks, vs,
             _on(table, "block_table", _I32, t_shape, dev)),
            (n_k, d, page, n_pages, _int(t_shape[1])), code)


def kv_write(k, v, k_pages, v_pages, block_table, start, count=None, k_scales=None,
             v_scales=None):
    """Write K, V [b, T, n_k, d] bf16 (columns of a fused projection's output will do) of T new tokens
    per sequence into the pages [n_pages, n_k, page, d] of a cache, bf16 or e4m3 (then with
    scale bytes [n_pages, n_k, page]): token t of sequence s at position start[s] + t, for
    t < count[s] (count None: all T).  Sequences with a negative start are skipped."""
    dev = _device(k, "k", 4)
    shape = k.shape
    b, T, n_k, d = shape
    ptrs, dims, code = _pages(k_pages, v_pages, k_scales, v_scales, block_table, b, dev)
    if dims[0] != n_k or dims[1] != d:
        raise ValueError("k and the pages disagree in shape")
    kp, k_row = _rows(k, "k", _BF, shape, dev)
    vp, v_row = _rows(v, "v", _BF, shape, dev)
    _call("basp_kv_write", (_lib or lib()).basp_kv_write, dev, kp, vp, *ptrs,
          _on(start, "start", _I32, (b,), dev),
          None if count is None else _on(count, "count", _I32, (b,), dev), b, T, *dims, k_row,
          v_row, code)


def kv_read(k_pages, v_pages, block_table, T: int, start=None, count=None, k_scales=None,
            v_scales=None, k=None, v=None):
    """Positions start[s] .. start[s] + count[s] - 1 of every sequence (start None: from 0, count None:
    T) out of a paged cache, as (k, v) [b, T, n_k, d] bf16; rows past count[s] are zeros."""
    dev = _device(block_table, "block_table", 2)
    b = block_table.shape[0]
    ptrs, dims, code = _pages(k_pages, v_pages, k_scales, v_scales, block_table, b, dev)
    shape = (b, T, dims[0], dims[1])
    if k is None:
        k = block_table.new_empty(shape, dtype=_BF)
        kp = k.data_ptr()
    else:
        kp = _on(k, "k", _BF, shape, dev)
    if v is None:
        v = torch.empty_like(k)
        vp = v.data_ptr()
    else:
        vp = _on(v, "v", _BF, shape, dev)
    _call("basp_kv_read", (_lib or lib()).basp_kv_read, dev, *ptrs,
          None if start is None else _on(start, "start", _I32, (b,), dev),
          None if count is None else _on(count, "count", _I32, (b,), dev), kp, vp, b, T, *dims,
          code)
    return k, v


def attn_decode_workspace_bytes(b, n_q, n_k, d, max_len) -> int:
    return int(lib().basp_attn_decode_workspace_bytes(b, n_q, n_k, d, max_len))


def attn_decode(q, k_pages, v_pages, block_table, lens, scale: float | None = None,
                max_len: int | None = None, k_scales=None, v_scales=None, out=None, lse=None,
                workspace=None):
    """Attention of one new token per sequence, q [b, n_q, d] bf16, over the first lens[s] tokens of
    a paged cache (the new token's own K, V written before, and counted): returns (o bf16 [b, n_q,
    d], lse fp32 [b, n_q]).  A length of 0 gives zeros and -inf.  ``max_len``: the longest sequence
    expected (default: all the table holds).  Two calls that may overlap on the device, captured
    graphs among them, need a ``workspace`` each (default: one of its own per call)."""
    dev = _device(q, "q", 3)
    shape = q.shape
    b, n_q, d = shape
    ptrs, dims, code = _pages(k_pages, v_pages, k_scales, v_scales, block_table, b, dev)
    n_k, dp, page, n_pages, max_pages = dims
    if dp != d:
        raise ValueError("q and the pages disagree in shape")
    if scale is None:
        scale = d ** -0.5
    max_len = _int(max_pages * page if max_len is None else max_len)
    qp, q_row = _rows(q, "q", _BF, shape, dev)
    if out is None:
        out = _like(q)
        op = out.data_ptr()
    else:
        op = _on(out, "out", _BF, shape, dev)
    if lse is None:
        lse = q.new_empty((b, n_q), dtype=_F32)
        lp = lse.data_ptr()
    else:
        lp = _on(lse, "lse", _F32, (b, n_q), dev)
    L = _lib or lib()
    need = 0 if workspace is not None else L.basp_attn_decode_workspace_bytes(b, n_q, n_k, d,
                                                                              max_len)
    workspace, ws, ws_n = _space(workspace, need, q, dev)
    _call("basp_attn_decode", L.basp_attn_decode, dev, qp, *ptrs, _on(lens, "lens", _I32, (b,), dev),
          op, lp, ws, ws_n, b, n_q, n_k, d, page, n_pages, max_pages, max_len, q_row, scale, code)
    return out, lse
