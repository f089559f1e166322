"""The paged key/value cache between the QKV and the output projection.

Names follow include/rrs.h without the prefix. The calls check their tensors, pass the device
pointers and the current HIP stream to librrs.so, and raise on a non-zero status, in a
compiled module (_torch_calls.so, csrc/rrs_torch.cpp): host time counts for calls that a decode
step makes once per layer. Every step of the computation runs in the library's kernels.

A call without `workspace` takes what it needs from torch's caching allocator, also under
torch.cuda.graph; under a capture that torch does not manage, pass one that outlives the graph.
"""
from __future__ import annotations

import importlib
import os
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

from ._binding import RRSError, lib

# Formats of the cached values (include/rrs.h, RRS_KV_*).
KV_F16 = 0
KV_INT4 = 1

_module = None


def _load():
    """The compiled calls (built by build.py)."""
    global _module
    lib()   # raises if librrs.so is missing
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_torch_calls.so")
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m "
                           "paper_2409_20361_amd.build` (there is no fallback)")
    module = importlib.import_module("._torch_calls", __package__)
    module.set_error(RRSError)
    _module = module
    return module


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
    return (_module or _load()).rope_kv_append(qkv, positions, rope, *cache, seq, slot, heads,
                                               sections, interleaved, weights, slot_pos, out)


def paged_attention_workspace_bytes(cache: KVCache, heads: int, max_length: int,
                                    with_weights: bool = False) -> int:
    return (_module or _load()).paged_attention_workspace_bytes(*cache, heads, max_length,
                                                                with_weights)


def paged_attention(Q: torch.Tensor, cache: KVCache, lengths: torch.Tensor,
                    max_length: Optional[int] = None, scale: Optional[float] = None,
                    mask: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
                    return_lse: bool = False, workspace: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None):
    """Attention of one new token per sequence over its cache.

    Q: sequences x heads x head dim fp16; lengths: (sequences,) int32, the new token included;
    max_length: a bound on them (None: the cache's capacity), by which the launches and the workspace are
    chosen, so best a tight one; scale: of the logits (None:
    head dim^-1/2); mask: (sequences, capacity) bool, False slots take no part; weights:
    (sequences, KV heads, capacity) float32, gains every slot's attention weight. Returns
    the output (as Q), or (output, lse) with lse (sequences, heads) float32."""
    return (_module or _load()).paged_attention(Q, *cache, lengths, max_length, scale, mask,
                                                weights, return_lse, workspace, out)


def kv_evict_workspace_bytes(cache: KVCache, max_length: int, budget: int) -> int:
    return (_module or _load()).kv_evict_workspace_bytes(*cache, max_length, budget)


def kv_evict(cache: KVCache, lengths: torch.Tensor, weights: torch.Tensor, slot_pos: torch.Tensor,
             keep_from: torch.Tensor, budget: int, max_length: Optional[int] = None, out=None,
             workspace: Optional[torch.Tensor] = None
             ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Brings every sequence down to its `budget` slots of largest weight, in place.

    weights, slot_pos: (sequences, KV heads, capacity) float32 / int32; keep_from: (sequences,)
    int32, tokens at positions from it on are kept first; max_length: a bound on the lengths (None: the
    cache's capacity), above 16384 with the launches for long rows. Returns (kept, lengths, weights,
    slot_pos) of the cache after the move (include/rrs.h, rrs_kv_evict), new tensors or `out`;
    none of them may overlap an input, the cache, the workspace or another."""
    return (_module or _load()).kv_evict(*cache, lengths, weights, slot_pos, keep_from, budget,
                                         max_length, out, workspace)


def kv_read(cache: KVCache, lengths: torch.Tensor, max_length: Optional[int] = None, out=None
            ) -> Tuple[torch.Tensor, torch.Tensor]:
    """The cached values as fp16: (K, V), each sequences x KV heads x max_length x head dim, zeros
    from a sequence's length on."""
    return (_module or _load()).kv_read(*cache, lengths, max_length, out)
