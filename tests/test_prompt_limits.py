"""Host-only checks of the sizes that prompt attention takes (no GPU needed; the pointers are never dereferenced): every
call within the documented number of workgroups gets past the size checks, to the one of the alignment."""
import ctypes

import pytest

import paper_2409_20361_amd as rrs
import test_kv_abi as A


def _call(D, sequences, kv_heads, heads, tokens, top):
    c = A._cache(head_dim=D, sequences=sequences, kv_heads=kv_heads)
    return rrs.lib().rrs_prompt_attention(A.MIS, tokens, heads, ctypes.byref(c), A.P, tokens, A.P, top, 0.1,
                                          None, A.P, None, A.P, 1 << 62, None)


@pytest.mark.parametrize("D,sequences,kv_heads,heads,tokens", [
    # r pairs, t tiles of 128 rows: r t < 2^24. An odd number of the tiles that a workgroup of eight waves takes two of
    (128, 5000000, 1, 1, 300), (128, 2500000, 2, 2, 300), (128, 1 << 22, 1, 1, 384), (128, 2900000, 1, 1, 640),
    # pairs that are no multiple of the eight XCDs
    (64, (1 << 23) - 1, 1, 1, 256), (256, (1 << 23) - 1, 1, 1, 256), (128, (1 << 23) - 1, 1, 1, 256),
    (64, 5592405, 1, 1, 384), (128, 1398101, 3, 3, 384)])
def test_within(D, sequences, kv_heads, heads, tokens):
    rows = tokens * heads // kv_heads
    assert rows > 128 and sequences * kv_heads * -(-rows // 128) < 1 << 24
    for top in (1, 80):
        assert _call(D, sequences, kv_heads, heads, tokens, top) == A.ALIGN


@pytest.mark.parametrize("D,sequences,kv_heads,heads,tokens", [
    (128, 1 << 22, 1, 1, 385), (64, 1 << 22, 1, 1, 512), (256, 5592406, 1, 1, 384), (128, 1 << 20, 4, 4, 512)])
def test_past(D, sequences, kv_heads, heads, tokens):
    rows = tokens * heads // kv_heads
    past = sequences * kv_heads * -(-rows // 128) >= 1 << 24
    for top in (1, 80):
        assert past and _call(D, sequences, kv_heads, heads, tokens, top) == A.SHAPE
