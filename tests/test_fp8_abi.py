"""Host-only checks of the FP8 cache: wrong arguments come back with the documented status before any device
is touched (no GPU needed; the pointers are never dereferenced)."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2409_20361_amd as rrs
import test_kv_abi as A

FP8 = rrs.KV_FP8


def _cache(**kw):
    return A._cache(**{**dict(format=FP8, k_scale=A.P, v_scale=A.P), **kw})


@pytest.mark.parametrize("call", [A._append, A._attend, A._evict, A._read])
@pytest.mark.parametrize("kw,want", [
    (dict(k_scale=None), A.NULL), (dict(v_scale=None), A.NULL), (dict(k=None), A.NULL),
    (dict(k_scale=A.MIS), A.ALIGN), (dict(v_scale=A.MIS), A.ALIGN), (dict(k=A.MIS), A.ALIGN),
    (dict(head_dim=96), A.SHAPE), (dict(page_size=8), A.SHAPE), (dict(pages=0), A.SHAPE)])
def test_caches(call, kw, want):
    # Eviction refuses the format before it looks at the alignment.
    if call is A._evict and want == A.ALIGN:
        want = A.FLAGS
    assert call(_cache(**kw)) == want


def test_no_eviction():
    assert A._evict(_cache()) == A.FLAGS
    q = rrs.lib().rrs_kv_evict_workspace_bytes
    long = dict(max_pages=5000, page_size=16)
    assert q(ctypes.byref(_cache(**long)), 40000, 7) == 0
    assert q(ctypes.byref(A._cache(**long)), 40000, 7) > 0


def test_workspace():
    q = rrs.lib().rrs_paged_attention_workspace_bytes
    c = _cache()
    need = q(ctypes.byref(c), 4, 80, 1)
    assert need > 0 and A._attend(c, weights=A.P, bytes=need - 1) == A.WS


@pytest.mark.parametrize("kw", [dict(M=1 << 24), dict(M=15800000), dict(M=767, heads=1 << 20)])
def test_grid(kw):
    a = dict(stride=(kw.get("heads", 4) + 4) * 128)
    assert A._append(_cache(), **{**a, **kw}) == A.SHAPE


B, HK, D, P, PAGES = 2, 2, 128, 32, 9


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
@pytest.mark.parametrize("name,shape,dtype,error", [
    ("k", (PAGES, HK, P, D), torch.float16, TypeError),
    ("v", (PAGES, HK, P, D), torch.float16, TypeError),
    ("v", (PAGES, HK, P, D + 1), torch.float8_e4m3fn, ValueError),
    ("k_scale", (PAGES, HK, P), torch.float16, ValueError),
    ("v_scale", (PAGES, HK, P // 16), torch.float32, TypeError),
    ("v_scale", None, None, TypeError)])
def test_tensors(name, shape, dtype, error):
    with FakeTensorMode():
        t = {"k": torch.empty((PAGES, HK, P, D), dtype=torch.float8_e4m3fn, device="cuda:0"),
             "v": torch.empty((PAGES, HK, P, D), dtype=torch.float8_e4m3fn, device="cuda:0"),
             "table": torch.empty((B, 4), dtype=torch.int32, device="cuda:0"),
             "k_scale": torch.empty((PAGES, HK, P // 16), dtype=torch.float16, device="cuda:0"),
             "v_scale": torch.empty((PAGES, HK, P // 16), dtype=torch.float16, device="cuda:0")}
        t[name] = torch.empty(shape, dtype=dtype, device="cuda:0") if shape else None
        lengths = torch.empty((B,), dtype=torch.int32, device="cuda:0")
        out = tuple(torch.empty((B, HK, 4 * P, D), dtype=torch.float16, device="cuda:0")
                    for _ in range(2))
    with pytest.raises(error):
        rrs.kv_read(rrs.KVCache(**t), lengths, out=out)


def test_empty_cache():
    table = torch.zeros((B, 4), dtype=torch.int32)
    cache = rrs.kv_cache(PAGES, HK, P, D, table, FP8)
    assert cache.k.dtype == torch.float8_e4m3fn and cache.k.shape == (PAGES, HK, P, D)
    assert cache.k_scale.shape == (PAGES, HK, P // 16) and not cache.k_scale.any()
    with pytest.raises(ValueError):
        rrs.kv_cache(PAGES, HK, P, D, table, 2)
