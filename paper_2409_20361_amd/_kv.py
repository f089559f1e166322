"""The paged key/value cache between the QKV and the output projection: ctypes marshalling.

Names follow include/rrs.h without the prefix. As in the layer's binding, every call checks its
tensors, passes their device pointers and the current HIP stream, and raises on a
non-zero status; every step of the computation runs in the library's kernels.
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

from ._binding import _check, _dev, _stream, lib

# Formats of the cached values (include/rrs.h, RRS_KV_*).
KV_F16 = 0
KV_INT4 = 1

_ROPE_INTERLEAVED = 1


class KVCache(NamedTuple):
    """One layer's cache. k, v: (pages, KV heads, page size, head dim) float16, or (..., head dim
    / 2) uint8 of packed INT4 codes with k_scale, v_scale (pages, KV heads, page size)
    float16; table: (sequences, pages per sequence) int32, sequence b's slot t being slot
    t % page size of page table[b, t // page size]."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None

    @property
    def capacity(self) -> int:
        """Slots of each sequence."""
        return self.table.shape[1] * self.k.shape[2]


# rrs_kv_cache: k, v, k_scale, v_scale, table, then format, pages, kv_heads, page_size, head_dim,
# sequences, max_pages (packing it takes a quarter of the time of a ctypes.Structure).
_pack = struct.Struct("5P7i4x").pack


def _kv(cache: KVCache):
    """(packed struct, KV heads, head dim, sequences, capacity) of a cache, its tensors checked."""
    k, v, table, k_scale, v_scale = cache
    shape = k.shape
    if len(shape) != 4 or table.dim() != 2:
        raise ValueError("cache: k must have 4 dimensions and table 2")
    pages, heads, P, width = shape
    B, per_seq = table.shape
    tp = _dev(table, "table", torch.int32, (B, per_seq))
    if k_scale is None and v_scale is None:
        kp, vp = _dev(k, "k", torch.float16, shape), _dev(v, "v", torch.float16, shape)
        return (_pack(kp, vp, 0, 0, tp, KV_F16, pages, heads, P, width, B, per_seq), heads, width,
                B, per_seq * P)
    kp, vp = _dev(k, "k", torch.uint8, shape), _dev(v, "v", torch.uint8, shape)
    ksp = _dev(k_scale, "k_scale", torch.float16, shape[:3])
    vsp = _dev(v_scale, "v_scale", torch.float16, shape[:3])
    return (_pack(kp, vp, ksp, vsp, tp, KV_INT4, pages, heads, P, 2 * width, B, per_seq), heads,
            2 * width, B, per_seq * P)


def _workspace(t: Optional[torch.Tensor], device: torch.device):
    """Pointer and bytes of a workspace (None: none)."""
    if t is None:
        return None, 0
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on {device}")
    return t.data_ptr(), t.numel() * t.element_size()


def kv_cache(pages: int, kv_heads: int, page_size: int, head_dim: int, table: torch.Tensor,
             format: int = KV_F16) -> KVCache:
    """An empty cache of one layer on the table's device."""
    dev = table.device
    if format == KV_F16:
        k, v = (torch.empty((pages, kv_heads, page_size, head_dim), dtype=torch.float16,
                            device=dev) for _ in range(2))
        return KVCache(k, v, table)
    if format != KV_INT4:
        raise ValueError("format must be KV_F16 or KV_INT4")
    k, v = (torch.empty((pages, kv_heads, page_size, head_dim // 2), dtype=torch.uint8, device=dev)
            for _ in range(2))
    ks, vs = (torch.empty((pages, kv_heads, page_size), dtype=torch.float16, device=dev)
              for _ in range(2))
    return KVCache(k, v, table, ks, vs)


def rope_table(positions: int, rotary_dim: int, theta: float = 10000.0,
               device: Union[str, torch.device] = "cuda") -> torch.Tensor:
    """(positions, rotary_dim) float32: cosines, then sines, of position p at the frequencies
    theta^(-2 j / rotary_dim), computed in float64 (a float32 angle is off by up to 2^-8
    at position 2^16)."""
    half = rotary_dim // 2
    inv = float(theta) ** (-torch.arange(half, dtype=torch.float64) / half)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def rope_kv_append(qkv: torch.Tensor, positions: torch.Tensor, rope: torch.Tensor, cache: KVCache,
                   seq: torch.Tensor, slot: torch.Tensor, heads: int,
                   sections: Optional[Sequence[int]] = None, interleaved: bool = False,
                   weights: Optional[torch.Tensor] = None,
                   slot_pos: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotates the queries and keys of qkv and appends keys and values to the cache.

    qkv: M x (heads + 2 KV heads) head dim fp16, as the QKV projection writes it (its rows may
    lie apart); positions: (M, axes) int32; rope: (positions, rotary dim) float32 (rope_table);
    sections: frequencies of each axis (None: all on the one axis); seq, slot: (M,) int32, the
    place of each token (out of range: not stored). weights, slot_pos: kv_evict's arrays;
    a stored token's entries become 0 and its position on axis 0. Returns the rotated queries,
    M x heads x head dim."""
    st, hk, D, B, capacity = _kv(cache)
    M = qkv.shape[0]
    width = (heads + 2 * hk) * D
    if (not qkv.is_cuda or qkv.dtype is not torch.float16 or qkv.dim() != 2
            or qkv.shape[1] != width or qkv.stride(1) != 1):
        raise ValueError(f"qkv must be a float16 GPU tensor (M, {width}) with unit column stride")
    stride = qkv.stride(0) if M > 1 else width
    axes = positions.shape[1] if positions.dim() == 2 else 0
    pp = _dev(positions, "positions", torch.int32, (M, axes))
    if rope.dim() != 2:
        raise ValueError("rope must have shape (positions, rotary dim)")
    rows, R = rope.shape
    rp = _dev(rope, "rope", torch.float32, (rows, R))
    sections = (R // 2,) if sections is None else tuple(sections)
    if len(sections) != axes:
        raise ValueError(f"sections must name {axes} axes, got {len(sections)}")
    sp, tp = _dev(seq, "seq", torch.int32, (M,)), _dev(slot, "slot", torch.int32, (M,))
    wp = None if weights is None else _dev(weights, "weights", torch.float32, (B, hk, capacity))
    op = None if slot_pos is None else _dev(slot_pos, "slot_pos", torch.int32, (B, hk, capacity))
    Q = out if out is not None else qkv.new_empty((M, heads, D))
    qp = _dev(Q, "out", torch.float16, (M, heads, D))
    _check(lib().rrs_rope_kv_append(
        qkv.data_ptr(), stride, M, heads, pp, axes, (ctypes.c_int32 * axes)(*sections), rp, rows,
        R, _ROPE_INTERLEAVED if interleaved else 0, st, sp, tp, qp, wp, op,
        _stream(qkv.device)), "rrs_rope_kv_append")
    return Q


def paged_attention_workspace_bytes(cache: KVCache, heads: int, max_length: int,
                                    with_weights: bool = False) -> int:
    return lib().rrs_paged_attention_workspace_bytes(_kv(cache)[0], heads,
                                                     max_length, int(with_weights))


def paged_attention(Q: torch.Tensor, cache: KVCache, lengths: torch.Tensor,
                    max_length: Optional[int] = None, scale: Optional[float] = None,
                    mask: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
                    return_lse: bool = False, workspace: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None):
    """Attention of one new token per sequence over its cache.

    Q: sequences x heads x head dim fp16; lengths: (sequences,) int32, the new token included;
    max_length: a bound on them (None: the cache's capacity); scale: of the logits (None:
    head dim^-1/2); mask: (sequences, capacity) bool, False slots take no part; weights:
    (sequences, KV heads, capacity) float32, gains every slot's attention weight. Returns
    the output (as Q), or (output, lse) with lse (sequences, heads) float32."""
    st, hk, D, B, capacity = _kv(cache)
    heads = Q.shape[1] if Q.dim() == 3 else 0
    qp = _dev(Q, "Q", torch.float16, (B, heads, D))
    lp = _dev(lengths, "lengths", torch.int32, (B,))
    if max_length is None:
        max_length = capacity
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    mp = None if mask is None else _dev(mask, "mask", torch.bool, (B, capacity))
    wp = None if weights is None else _dev(weights, "weights", torch.float32, (B, hk, capacity))
    Y = out if out is not None else torch.empty_like(Q)
    yp = _dev(Y, "out", torch.float16, (B, heads, D))
    lse = torch.empty((B, heads), dtype=torch.float32, device=Q.device) if return_lse else None
    if workspace is None:
        need = lib().rrs_paged_attention_workspace_bytes(st, heads, max_length, wp is not None)
        if need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=Q.device)
    wsp, wsb = _workspace(workspace, Q.device)
    _check(lib().rrs_paged_attention(qp, heads, st, lp, max_length, scale, mp, wp, yp,
                                     None if lse is None else lse.data_ptr(), wsp, wsb,
                                     _stream(Q.device)), "rrs_paged_attention")
    return Y if lse is None else (Y, lse)


def kv_evict_workspace_bytes(cache: KVCache, max_length: int, budget: int) -> int:
    return lib().rrs_kv_evict_workspace_bytes(_kv(cache)[0], max_length, budget)


def kv_evict(cache: KVCache, lengths: torch.Tensor, weights: torch.Tensor, slot_pos: torch.Tensor,
             keep_from: torch.Tensor, budget: int, max_length: Optional[int] = None, out=None,
             workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Brings every sequence down to its `budget` slots of largest weight, in place.

    weights, slot_pos: (sequences, KV heads, capacity) float32 / int32; keep_from: (sequences,)
    int32, tokens at positions from it on are kept first. Returns (kept, lengths, weights,
    slot_pos) of the cache after the move (include/rrs.h, rrs_kv_evict), new tensors or `out`;
    none of them may be an input."""
    st, hk, D, B, capacity = _kv(cache)
    lp = _dev(lengths, "lengths", torch.int32, (B,))
    wp = _dev(weights, "weights", torch.float32, (B, hk, capacity))
    pp = _dev(slot_pos, "slot_pos", torch.int32, (B, hk, capacity))
    fp = _dev(keep_from, "keep_from", torch.int32, (B,))
    if max_length is None:
        max_length = capacity
    if not 1 <= budget <= capacity:
        raise ValueError(f"budget must be in [1, {capacity}], got {budget}")
    if out is None:
        out = (lengths.new_empty((B, hk, budget)), torch.empty_like(lengths),
               torch.empty_like(weights), torch.empty_like(slot_pos))
    kept, new, w2, p2 = out
    kp = _dev(kept, "kept", torch.int32, (B, hk, budget))
    np_ = _dev(new, "new_lengths", torch.int32, (B,))
    w2p = _dev(w2, "weights_out", torch.float32, (B, hk, capacity))
    p2p = _dev(p2, "pos_out", torch.int32, (B, hk, capacity))
    if w2p == wp or p2p == pp or np_ == lp:
        raise ValueError("kv_evict: outputs must not be inputs")
    if workspace is None:
        need = lib().rrs_kv_evict_workspace_bytes(st, max_length, budget)
        if need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=lengths.device)
    wsp, wsb = _workspace(workspace, lengths.device)
    _check(lib().rrs_kv_evict(st, lp, max_length, wp, pp, fp, budget, kp, np_, w2p, p2p, wsp, wsb,
                              _stream(lengths.device)), "rrs_kv_evict")
    return kept, new, w2, p2


def kv_read(cache: KVCache, lengths: torch.Tensor, max_length: Optional[int] = None, out=None
            ) -> Tuple[torch.Tensor, torch.Tensor]:
    """The cached values as fp16: (K, V), each sequences x KV heads x max_length x head dim, zeros
    from a sequence's length on."""
    st, hk, D, B, capacity = _kv(cache)
    lp = _dev(lengths, "lengths", torch.int32, (B,))
    if max_length is None:
        max_length = capacity
    if not 1 <= max_length <= capacity:
        raise ValueError(f"max_length must be in [1, {capacity}], got {max_length}")
    if out is None:
        out = tuple(torch.empty((B, hk, max_length, D), dtype=torch.float16,
                                device=lengths.device) for _ in range(2))
    K, V = out
    kp = _dev(K, "K", torch.float16, (B, hk, max_length, D))
    vp = _dev(V, "V", torch.float16, (B, hk, max_length, D))
    _check(lib().rrs_kv_read(st, lp, max_length, kp, vp, _stream(lengths.device)),
           "rrs_kv_read")
    return K, V
