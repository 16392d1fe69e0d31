"""One rank's share of a batch-aware Ulysses attention layer, on one GPU.

A rank of a BASP group (G members, Sec. IV of the paper) receives G sequence
shards of Q, K, V, runs attention on its H/G query heads over the full
sequence, and returns the output to the G shard owners; the backward mirrors
this with dO in and dQ, dK, dV out (the transposed exchanges of Ulysses,
Sec. II-C).  `RankShare` holds every device buffer of that share, allocated
once, and chains the library calls:

  forward:  pack(Q), pack(K), pack(V) -> attn_fwd -> unpack(O)
  backward: pack(dO) -> attn_bwd -> unpack(dQ), unpack(dK), unpack(dV)

(the three packs and the three gradient unpacks each as one call,
pack_qkv / unpack_grads).  A step is the forward, then the backward: dO is
packed only after O has left, as in training, where dO follows from O.

With fewer kv heads than members (H_kv < G, G divisible by H_kv) the rank
holds one kv head shared by G/H_kv members, and its dK, dV are that head's
partial gradients: they are added into the shards (unpack_add), so the dK/dV
shard buffers accumulate over repeated backward calls.

The exchange itself (RCCL all-to-all) is outside this share: the shard
buffers stand for the receive and send buffers of that exchange.

`forward_sharded` / `backward_sharded` run the same step with no pack or
unpack pass: attention reads the shard buffers in place and writes O, dQ,
dK, dV straight into the send buffers (bit for bit the same results); with a
shared kv head, dK and dV go to one send block per member (`dk_send`,
`dv_send`), each the member's partial gradient for that member's tokens.

With a `QkNormRope` the share's Q and K are normalised per head and rotated
between the pack and attention, and the backward goes through both:

  forward:  pack(Q, K, V) -> qk_norm_rope -> attn_fwd -> unpack(O)
  backward: pack(dO) -> attn_bwd -> qk_norm_rope_bwd -> unpack(dQ, dK, dV)

`dq_weight`, `dk_weight` are then the rank's parts of the weights' gradients
(those of its heads), to be summed over the group.  Attention on the shard
buffers in place has no such step: there the owner of a shard calls
qk_norm_rope on it before the exchange.

With a `ScoreRule` attention is that of packed documents, prefixes and padding, with scores
capped and biased by distance, forward (`attn_span_fwd`), backward (`attn_span_bwd`) and in
`decode`.  It needs the rank's tensors packed, as the norm does.

After a forward, either one, `fill_cache` puts the prompt's K and V into a paged
cache, and `decode` takes the share on by one token per sequence.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import (attn_bwd, attn_bwd_sharded, attn_bwd_sharded_workspace_bytes,
               attn_bwd_workspace_bytes, attn_fwd,
               attn_fwd_sharded, attn_span_bwd, attn_span_bwd_workspace_bytes, attn_span_fwd,
               heads_per_member, pack, pack_qkv, qk_norm_rope, qk_norm_rope_bwd,
               qk_norm_rope_bwd_workspace_bytes, unpack, unpack_add, unpack_grads)


@dataclass
class QkNormRope:
    """Norm weights (fp32 [d], both None: no norm) and position tables (`rope_table`, both None: no
    rotation) of a layer's queries and keys."""
    q_weight: torch.Tensor | None
    k_weight: torch.Tensor | None
    cos: torch.Tensor | None
    sin: torch.Tensor | None
    eps: float = 1e-6
    interleaved: bool = False


@dataclass
class ScoreRule:
    """What a layer's attention does to its scores: which keys each token sees (`attn_spans`, int32
    [b, S, 2]; None: causal), the cap (None: none), and the slopes of all H query heads (fp32 [H];
    None: no bias), of which a rank takes its own.  `decode` has the cap and slopes; its tokens see all
    cached ones, whatever the spans."""
    spans: torch.Tensor | None = None
    cap: float | None = None
    slopes: torch.Tensor | None = None


class RankShare:
    def __init__(self, q_shards, k_shards, v_shards, do_shards, G: int, rank: int,
                 scale: float | None = None, norm_rope: QkNormRope | None = None,
                 rule: ScoreRule | None = None):
        self.G, self.rank = G, rank
        self.q_shards, self.k_shards, self.v_shards = q_shards, k_shards, v_shards
        self.do_shards = do_shards
        b, Sg, H, d = q_shards[0].shape
        H_kv = k_shards[0].shape[2]
        self.b, self.S, self.H, self.H_kv, self.d = b, Sg * G, H, H_kv, d
        self.Hl, self.Hkl = H // G, heads_per_member(H_kv, G)
        self.shared_kv = H_kv < G
        self.scale = d ** -0.5 if scale is None else scale
        dev = q_shards[0].device
        bf, f32 = torch.bfloat16, torch.float32
        S = self.S
        # head-sharded local tensors
        self.q = torch.empty((b, S, self.Hl, d), dtype=bf, device=dev)
        self.k = torch.empty((b, S, self.Hkl, d), dtype=bf, device=dev)
        self.v = torch.empty_like(self.k)
        self.o = torch.empty_like(self.q)
        self.lse = torch.empty((b, self.Hl, S), dtype=f32, device=dev)
        self.do = torch.empty_like(self.q)
        self.dq = torch.empty((b, S, self.Hl, d), dtype=f32, device=dev)
        self.dk = torch.empty((b, S, self.Hkl, d), dtype=f32, device=dev)
        self.dv = torch.empty_like(self.dk)
        # send buffers of the output exchanges (shard layout)
        self.o_shards = [torch.zeros((b, Sg, H, d), dtype=bf, device=dev) for _ in range(G)]
        self.dq_shards = [torch.zeros((b, Sg, H, d), dtype=f32, device=dev) for _ in range(G)]
        self.dk_shards = [torch.zeros((b, Sg, H_kv, d), dtype=f32, device=dev) for _ in range(G)]
        self.dv_shards = [torch.zeros((b, Sg, H_kv, d), dtype=f32, device=dev) for _ in range(G)]
        # in-place backward with a shared kv head: the partial dK, dV go to
        # one send block per member (the reverse exchange sums them)
        if self.shared_kv:
            self.dk_send = [torch.zeros((b, Sg, 1, d), dtype=f32, device=dev) for _ in range(G)]
            self.dv_send = [torch.zeros((b, Sg, 1, d), dtype=f32, device=dev) for _ in range(G)]
        ws = max(attn_bwd_workspace_bytes(b, S, H, H_kv, d, G),
                 attn_bwd_sharded_workspace_bytes(b, S, H, H_kv, d, G))
        # norm and rotation: what the pack gives, kept for the backward; the
        # weights' gradients (this rank's heads' part)
        self.norm_rope = norm_rope
        self.q_in, self.k_in = self.q, self.k
        self.dq_weight = self.dk_weight = None
        if norm_rope is not None:
            self.q_in, self.k_in = torch.empty_like(self.q), torch.empty_like(self.k)
            if norm_rope.q_weight is not None:
                self.dq_weight = torch.empty_like(norm_rope.q_weight)
                self.dk_weight = torch.empty_like(norm_rope.k_weight)
                ws = max(ws, qk_norm_rope_bwd_workspace_bytes(b, S, self.Hl, self.Hkl, d))
        self.rule = rule
        self.slopes = None
        if rule is not None:
            if rule.slopes is not None:
                if rule.slopes.shape != (H,):
                    raise ValueError(f"slopes must be those of all {H} query heads")
                self.slopes = rule.slopes[rank * self.Hl:(rank + 1) * self.Hl].contiguous()
            ws = max(ws, attn_span_bwd_workspace_bytes(b, S, self.Hl, self.Hkl, d))
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=dev)
        # where the last forward's K and V are: "local" (k, v), "shards", or in neither
        self._kv = None

    # individual steps, so that callers can time them
    def pack_qkv(self):
        pack_qkv(self.q_shards, self.k_shards, self.v_shards, self.rank, q=self.q_in, k=self.k_in,
                 v=self.v)
        self._kv = "local" if self.norm_rope is None else None

    def qk_norm_rope(self):
        n = self.norm_rope
        qk_norm_rope(self.q_in, self.k_in, n.q_weight, n.k_weight, n.cos, n.sin, eps=n.eps,
                     interleaved=n.interleaved, q_out=self.q, k_out=self.k)
        self._kv = "local"

    def _rule(self):
        return {"scale": self.scale, "cap": self.rule.cap, "slopes": self.slopes}

    def attn_fwd(self):
        if self.rule is not None:
            attn_span_fwd(self.q, self.k, self.v, self.rule.spans, out=self.o, lse=self.lse,
                          **self._rule())
            return
        attn_fwd(self.q, self.k, self.v, G=self.G, scale=self.scale, out=self.o, lse=self.lse,
                 H_kv=self.H_kv)

    def unpack_o(self):
        unpack(self.o, self.o_shards, self.rank)

    def pack_do(self):
        pack(self.do_shards, self.rank, out=self.do)

    def attn_bwd(self):
        if self.rule is not None:
            attn_span_bwd(self.q, self.k, self.v, self.o, self.lse, self.do, self.rule.spans,
                          dq=self.dq, dk=self.dk, dv=self.dv, workspace=self.workspace,
                          **self._rule())
            return
        attn_bwd(self.q, self.k, self.v, self.o, self.lse, self.do, G=self.G, scale=self.scale,
                 dq=self.dq, dk=self.dk, dv=self.dv, workspace=self.workspace, H_kv=self.H_kv)

    def qk_norm_rope_bwd(self):
        """dq, dk in place: from the gradients of attention's Q and K to those of the packed ones."""
        n = self.norm_rope
        qk_norm_rope_bwd(self.q_in, self.k_in, self.dq, self.dk, n.q_weight, n.k_weight, n.cos, n.sin,
                         eps=n.eps, interleaved=n.interleaved, dq=self.dq, dk=self.dk,
                         dq_weight=self.dq_weight, dk_weight=self.dk_weight,
                         workspace=self.workspace)

    def _unpack_kv_grad(self, local, shards):
        (unpack_add if self.shared_kv else unpack)(local, shards, self.rank)

    def unpack_grads(self):
        unpack_grads(self.dq, self.dk, self.dv, self.dq_shards, self.dk_shards, self.dv_shards,
                     self.rank)

    def forward(self):
        self.pack_qkv()
        if self.norm_rope is not None:
            self.qk_norm_rope()
        self._kv = "local"
        self.attn_fwd()
        self.unpack_o()

    def backward(self):
        self.pack_do()
        self.attn_bwd()
        if self.norm_rope is not None:
            self.qk_norm_rope_bwd()
        self.unpack_grads()

    def step(self):
        self.forward()
        self.backward()

    # generation after the prompt
    def fill_cache(self, cache, block_table):
        """K and V of the last forward into a `PagedKV`, sequence s's tokens from position 0 on in the
        pages that row s of the block table lists.  After `forward_sharded` the rank's head is read
        from the shard buffers, which must still hold that forward's K and V.  The last forward is
        the one that Python called last: the replay of a captured one does not count."""
        if self._kv is None:
            raise RuntimeError("fill_cache takes K and V of a forward: call one first")
        dev, i32 = self.k.device, torch.int32
        if self._kv == "local":
            cache.write(self.k, self.v, block_table, torch.zeros(self.b, dtype=i32, device=dev))
            return
        Sg, h = self.S // self.G, self.rank * self.H_kv // self.G
        first = Sg * torch.arange(self.G, dtype=i32, device=dev)  # token of each shard
        start = first[:, None].expand(self.G, self.b).contiguous()
        for k, v, at in zip(self.k_shards, self.v_shards, start):
            cache.write(k[:, :, h:h + self.Hkl], v[:, :, h:h + self.Hkl], block_table, at)

    def decode(self, cache, q, k, v, block_table, lens, max_len: int | None = None, workspace=None,
               groups=None, prefix_lens=None):
        """One new token per sequence: q [n, 1, H/G, d] and k, v [n, 1, Hkl, d], the rank's heads of
        its projections, at position lens[s] - 1.  Norm and rotation if the share has them, the
        token's K and V into the cache, and attention over the lens[s] tokens, with the share's cap
        and slopes if it has them: returns (O [n, H/G, d], LSE [n, H/G]).  A length of 0 is a slot
        without a sequence.  ``groups``, ``prefix_lens``: sequences that share a prefix, in pages
        that no new token goes to (`attn_decode_shared`)."""
        at = lens - 1
        n = self.norm_rope
        if n is not None:
            q, k = qk_norm_rope(q, k, n.q_weight, n.k_weight, n.cos, n.sin, eps=n.eps,
                                interleaved=n.interleaved, positions=at.view(-1, 1))
        cache.write(k, v, block_table, at)
        if self.rule is not None or groups is not None or prefix_lens is not None:
            rule = {"scale": self.scale} if self.rule is None else self._rule()
            return cache.attend_shared(q[:, 0], block_table, lens, groups, prefix_lens,
                                       max_len=max_len, workspace=workspace, **rule)
        return cache.attend(q[:, 0], block_table, lens, scale=self.scale, max_len=max_len,
                            workspace=workspace)

    # attention on the shard buffers in place
    def _check_in_place(self):
        if self.norm_rope is not None:
            raise ValueError("attention in place takes normalised, rotated shards: call qk_norm_rope "
                             "on them before the exchange")
        if self.rule is not None:
            raise ValueError("attention in place is causal: a share with a ScoreRule packs")

    def forward_sharded(self):
        self._check_in_place()
        attn_fwd_sharded(self.q_shards, self.k_shards, self.v_shards, self.o_shards, self.rank,
                         scale=self.scale, lse=self.lse)
        self._kv = "shards"

    def backward_sharded(self):
        self._check_in_place()
        dk, dv = ((self.dk_send, self.dv_send) if self.shared_kv
                  else (self.dk_shards, self.dv_shards))
        attn_bwd_sharded(self.q_shards, self.k_shards, self.v_shards, self.o_shards, self.lse,
                         self.do_shards, self.dq_shards, dk, dv, self.rank, scale=self.scale,
                         workspace=self.workspace)

    def step_sharded(self):
        self.forward_sharded()
        self.backward_sharded()

    # work counts (FlashAttention convention: causal half of S^2)
    def attn_fwd_flops(self) -> float:
        return 2.0 * self.b * self.Hl * self.d * float(self.S) ** 2

    def attn_bwd_flops(self) -> float:
        return 2.5 * self.attn_fwd_flops()

    def step_permutation_calls(self) -> list:
        """(name, call, bytes read + written) of the four pack/unpack calls a step makes."""
        nb = self.pack_unpack_bytes()
        return [("pack_qkv", self.pack_qkv, nb["pack_qkv"]),
                ("unpack_o", self.unpack_o, nb["unpack_o"]),
                ("pack_do", self.pack_do, nb["pack_do"]),
                ("unpack_grads", self.unpack_grads, nb["unpack_grads"])]

    def permutation_calls(self) -> list:
        """(name, call, bytes read + written) of each of the eight single-tensor permutations."""
        two = lambda t: 2 * t.numel() * t.element_size()
        # an added gradient is read on both sides and written once
        kv_grad = (lambda t: 3 * t.numel() * t.element_size()) if self.shared_kv else two
        return [
            ("pack_q", lambda: pack(self.q_shards, self.rank, out=self.q_in), two(self.q)),
            ("pack_k", lambda: pack(self.k_shards, self.rank, out=self.k_in), two(self.k)),
            ("pack_v", lambda: pack(self.v_shards, self.rank, out=self.v), two(self.v)),
            ("unpack_o", lambda: unpack(self.o, self.o_shards, self.rank), two(self.o)),
            ("pack_do", lambda: pack(self.do_shards, self.rank, out=self.do), two(self.do)),
            ("unpack_dq", lambda: unpack(self.dq, self.dq_shards, self.rank), two(self.dq)),
            ("unpack_dk", lambda: self._unpack_kv_grad(self.dk, self.dk_shards), kv_grad(self.dk)),
            ("unpack_dv", lambda: self._unpack_kv_grad(self.dv, self.dv_shards), kv_grad(self.dv)),
        ]

    def pack_unpack_bytes(self) -> dict:
        """Bytes read + written by each permutation (each moved element twice)."""
        bq = self.q.numel() * 2
        bkv = self.k.numel() * 2
        return {
            "pack_qkv": 2 * (bq + 2 * bkv),
            "unpack_o": 2 * bq,
            "pack_do": 2 * bq,
            "unpack_grads": (2 * self.dq.numel() + (3 if self.shared_kv else 2) * 2 * self.dk.numel()) * 4,
        }
