"""Host-only checks of the key/value cache's C ABI (no GPU needed): wrong arguments come back with
the documented status before any device is touched. The pointers are never dereferenced."""
import ctypes

import pytest

import paper_2409_20361_amd as rrs


class _Struct(ctypes.Structure):   # rrs_kv_cache
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "table")] + [
        (n, ctypes.c_int32) for n in ("format", "pages", "kv_heads", "page_size", "head_dim",
                                      "sequences", "max_pages")]

NULL, SHAPE, ALIGN, WS, FLAGS = -1, -2, -4, -5, -9
P, MIS = 0x10000, 0x10004


def _cache(**kw):
    a = dict(k=P, v=P, k_scale=None, v_scale=None, table=P, format=0, pages=4, kv_heads=2,
             page_size=16, head_dim=128, sequences=3, max_pages=5)
    a.update(kw)
    return _Struct(*(a[n] for n, _ in _Struct._fields_))


BAD_CACHES = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL),
    (dict(format=1), NULL), (dict(format=1, k_scale=P), NULL),
    (dict(head_dim=96), SHAPE), (dict(head_dim=512), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=48), SHAPE), (dict(page_size=512), SHAPE), (dict(pages=0), SHAPE),
    (dict(kv_heads=0), SHAPE), (dict(sequences=0), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(sequences=1 << 23, kv_heads=1), SHAPE), (dict(max_pages=1 << 27), SHAPE),
    (dict(max_pages=(1 << 26) + 1), SHAPE),
    (dict(format=2), FLAGS), (dict(format=-1), FLAGS),
    (dict(k=MIS), ALIGN), (dict(v=MIS), ALIGN), (dict(table=MIS), ALIGN),
    (dict(format=1, k_scale=MIS, v_scale=P), ALIGN),
    (dict(format=1, k_scale=P, v_scale=MIS), ALIGN),
]


def _append(cache=None, split=(64,), **kw):
    keep = (ctypes.c_int32 * 4)(*split)
    a = dict(qkv=P, stride=8 * 128, M=3, heads=4, pos=P, axes=len(split),
             sections=ctypes.addressof(keep), rope=P, rows=9, R=128, flags=0,
             cache=ctypes.byref(cache or _cache()), seq=P, slot=P, Q=P, weights=None,
             slot_pos=None)
    a.update(kw)
    return rrs.lib().rrs_rope_kv_append(*a.values(), None)


def _attend(cache=None, **kw):
    a = dict(Q=P, heads=4, cache=ctypes.byref(cache or _cache()), lengths=P, top=80, scale=0.1,
             mask=None, weights=None, out=P, lse=None, ws=P, bytes=1 << 40)
    a.update(kw)
    return rrs.lib().rrs_paged_attention(*a.values(), None)


def _evict(cache=None, **kw):
    a = dict(cache=ctypes.byref(cache or _cache()), lengths=P, top=80, w=P, pos=P, keep=P,
             budget=7, kept=P, new=P, w2=P, pos2=P, ws=None, bytes=0)
    a.update(kw)
    return rrs.lib().rrs_kv_evict(*a.values(), None)


def _read(cache=None, **kw):
    a = dict(cache=ctypes.byref(cache or _cache()), lengths=P, top=80, K=P, V=P)
    a.update(kw)
    return rrs.lib().rrs_kv_read(*a.values(), None)


@pytest.mark.parametrize("call", [_append, _attend, _evict, _read])
def test_caches(call):
    for kw, want in BAD_CACHES:
        assert call(_cache(**kw)) == want, kw


def test_null_struct():
    assert rrs.lib().rrs_kv_read(None, P, 80, P, P, None) == NULL
    assert rrs.lib().rrs_paged_attention_workspace_bytes(None, 4, 80, 0) == 0


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, NULL) for n in ("qkv", "pos", "rope", "seq", "slot", "Q", "sections")],
    (dict(M=0), SHAPE), (dict(heads=0), SHAPE), (dict(rows=0), SHAPE), (dict(R=0), SHAPE),
    (dict(R=120), SHAPE), (dict(R=144), SHAPE), (dict(R=64), SHAPE), (dict(axes=0), SHAPE),
    (dict(axes=5), SHAPE), (dict(stride=1016), SHAPE), (dict(stride=1028), SHAPE),
    (dict(flags=2), FLAGS),
    *[({n: MIS}, ALIGN) for n in ("qkv", "pos", "rope", "seq", "slot", "Q", "weights",
                                  "slot_pos")],
])
def test_append(kw, want):
    assert _append(**kw) == want


def test_append_sections():
    assert _append(split=(32, 31)) == SHAPE
    assert _append(split=(65, -1)) == SHAPE
    assert _append(split=(2 ** 31 - 1, 2 ** 31 - 1, 66)) == SHAPE


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, NULL) for n in ("Q", "lengths", "out")],
    (dict(heads=0), SHAPE), (dict(heads=3), SHAPE), (dict(heads=1 << 22), SHAPE),
    (dict(top=0), SHAPE), (dict(top=81), SHAPE),
    *[({n: MIS}, ALIGN) for n in ("Q", "lengths", "out", "mask", "weights", "lse", "ws")],
    (dict(weights=P, ws=None), NULL), (dict(weights=P, bytes=0), WS),
    *[(dict(scale=x), FLAGS) for x in (float("nan"), float("inf"), -float("inf"))],
])
def test_attend(kw, want):
    assert _attend(**kw) == want


def test_attend_workspace():
    q = rrs.lib().rrs_paged_attention_workspace_bytes
    c = _cache()
    need = q(ctypes.byref(c), 4, 80, 1)
    assert need > 0 and _attend(weights=P, bytes=need - 1) == WS
    for heads, top in ((0, 80), (3, 80), (4, 0), (4, 81)):
        assert q(ctypes.byref(c), heads, top, 1) == 0
    assert q(ctypes.byref(_cache(head_dim=100)), 4, 80, 1) == 0


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, NULL) for n in ("lengths", "w", "pos", "keep", "kept", "new", "w2", "pos2")],
    (dict(top=0), SHAPE), (dict(top=81), SHAPE), (dict(budget=0), SHAPE),
    (dict(budget=81), SHAPE),
    *[({n: MIS}, ALIGN) for n in ("lengths", "w", "pos", "keep", "kept", "new", "w2", "pos2")],
])
def test_evict(kw, want):
    assert _evict(**kw) == want


def test_evict_workspace():
    q = rrs.lib().rrs_kv_evict_workspace_bytes
    assert q(ctypes.byref(_cache()), 80, 7) == 0   # few slots: none
    c = _cache(max_pages=2000)
    assert q(ctypes.byref(c), 16384, 7) == 0
    need = q(ctypes.byref(c), 20000, 7)
    assert need > 0
    assert _evict(c, top=20000, ws=None, bytes=need) == NULL
    assert _evict(c, top=20000, ws=MIS, bytes=need) == ALIGN
    assert _evict(c, top=20000, ws=P, bytes=need - 1) == WS
    for top, budget in ((0, 7), (32001, 7), (20000, 0), (20000, 32001)):
        assert q(ctypes.byref(c), top, budget) == 0


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, NULL) for n in ("lengths", "K", "V")],
    (dict(top=0), SHAPE), (dict(top=81), SHAPE),
    *[({n: MIS}, ALIGN) for n in ("lengths", "K", "V")],
])
def test_read(kw, want):
    assert _read(**kw) == want
