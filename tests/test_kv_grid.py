"""Calls whose launches would be too large are refused before anything is enqueued (no GPU needed).

Sizes just within a limit are told from refused ones by a misaligned pointer, which is checked
later: no call here gets as far as a launch."""
import ctypes

import pytest

import paper_2409_20361_amd as rrs
from test_kv_abi import ALIGN, MIS, SHAPE, P, _append, _attend, _cache, _evict, _read

K16 = 1 << 14


@pytest.mark.parametrize("M,want", [((1 << 24) - 1, ALIGN), (1 << 24, SHAPE)])
def test_append(M, want):
    assert _append(M=M, qkv=MIS) == want


@pytest.mark.parametrize("sequences,budget,want", [
    ((1 << 22) - 1, 7, ALIGN), (1 << 22, 7, SHAPE), ((1 << 23) - 1, 80, SHAPE)])
def test_evict_selection(sequences, budget, want):
    c = _cache(sequences=sequences, kv_heads=1)
    assert _evict(c, budget=budget, lengths=MIS) == want


@pytest.mark.parametrize("top,budget,want", [
    # rows of 256 bytes, 16 to a workgroup
    (K16, 512 * 16, ALIGN), (K16, 512 * 16 + 1, SHAPE),   # slots below the budget
    (K16 + 9, 512 * 16, ALIGN),                           # moves: min(budget, top - budget)
    (2 * K16, 512 * 16 + 1, SHAPE), (2 * K16, 2 * K16 - 9, ALIGN)])
def test_evict_moves(top, budget, want):
    c = _cache(sequences=(1 << 15) - 1, kv_heads=1, max_pages=1 << 11)
    ws = dict(ws=P, bytes=1 << 62)
    assert _evict(c, top=top, budget=budget, lengths=MIS, **ws) == want
    n = rrs.lib().rrs_kv_evict_workspace_bytes(ctypes.byref(c), top, budget)
    assert (n > 0) == (want == ALIGN and top > K16)


@pytest.mark.parametrize("segments,want", [(31, ALIGN), (33, SHAPE)])
def test_evict_segments(segments, want):
    c = _cache(sequences=1 << 17, kv_heads=1, max_pages=1 << 15)
    assert _evict(c, top=segments * 8192, budget=1, lengths=MIS, ws=P, bytes=1 << 62) == want


@pytest.mark.parametrize("heads,top,weights,want", [
    (17, 63 * 1024, P, ALIGN), (17, 63 * 1024 + 1, P, SHAPE), (17, 1 << 19, None, ALIGN),
    (16, 1 << 19, P, ALIGN)])
def test_attend(heads, top, weights, want):
    # 2^18 sequences that stay whole: with more than 16 heads per KV head the weights take a second launch,
    # a workgroup per 1024 slots
    c = _cache(sequences=1 << 18, kv_heads=1, max_pages=1 << 15)
    assert _attend(c, heads=heads, top=top, weights=weights, lengths=MIS, bytes=1 << 62) == want
    n = rrs.lib().rrs_paged_attention_workspace_bytes(ctypes.byref(c), heads, top,
                                                      weights is not None)
    assert weights is None or (n > 0) == (want == ALIGN)


@pytest.mark.parametrize("top,want", [((1 << 23) - 2048, ALIGN), ((1 << 23) - 2047, SHAPE)])
def test_attend_cut(top, want):
    # 256 sequences of 8 heads that are cut: 2048 workgroups join, 2048 per 1024 slots add weights
    c = _cache(sequences=256, kv_heads=8, max_pages=1 << 19)
    assert _attend(c, heads=8, top=top, weights=P, lengths=MIS, bytes=1 << 62) == want


@pytest.mark.parametrize("top,want", [((1 << 14) - 16, ALIGN), ((1 << 14) - 15, SHAPE)])
def test_read(top, want):
    # 2^14 (sequence, KV head) pairs of head dim 128: 16 rows to a workgroup
    c = _cache(sequences=1 << 11, kv_heads=8, max_pages=1 << 11)
    assert _read(c, top=top, lengths=MIS) == want
