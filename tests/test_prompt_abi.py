"""Host-only checks of prompt attention: wrong arguments come back with the documented status, or are refused,
before any device is touched (no GPU needed; the pointers are never dereferenced)."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2409_20361_amd as rrs
import test_kv_abi as A

P, MIS = A.P, A.MIS


def _call(cache=None, **kw):
    a = dict(Q=P, M=20, heads=4, cache=ctypes.byref(cache or A._cache()), row_start=P, tokens=20,
             lengths=P, top=80, scale=0.1, mask=None, out=P, lse=None, ws=P, bytes=1 << 40)
    a.update(kw)
    return rrs.lib().rrs_prompt_attention(*a.values(), None)


def test_caches():
    for kw, want in A.BAD_CACHES:
        assert _call(A._cache(**kw)) == want, kw


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, A.NULL) for n in ("Q", "row_start", "lengths", "out")],
    (dict(heads=0), A.SHAPE), (dict(heads=3), A.SHAPE), (dict(heads=1 << 22), A.SHAPE),
    (dict(M=0), A.SHAPE), (dict(tokens=0), A.SHAPE), (dict(tokens=21), A.SHAPE),
    (dict(top=0), A.SHAPE), (dict(top=81), A.SHAPE),
    (dict(M=1 << 30, tokens=1 << 30), A.SHAPE),   # 2^31 rows to a KV head
    (dict(M=1 << 29, tokens=1 << 29), A.SHAPE),   # 2^25 workgroups
    *[({n: MIS}, A.ALIGN) for n in ("Q", "row_start", "lengths", "mask", "out", "lse", "ws")],
    *[(dict(scale=x), A.FLAGS) for x in (float("nan"), float("inf"), -float("inf"))]])
def test_arguments(kw, want):
    assert _call(**kw) == want


def test_workspace():
    q = rrs.lib().rrs_prompt_attention_workspace_bytes
    c = A._cache(max_pages=100, page_size=64)
    need = q(ctypes.byref(c), 4, 20, 6400)
    assert need > 0
    assert _call(c, top=6400, bytes=need - 1) == A.WS
    assert _call(c, top=6400, ws=None) == A.NULL
    for heads, tokens, top in ((0, 20, 80), (3, 20, 80), (4, 0, 80), (4, 20, 0), (4, 20, 6401)):
        assert q(ctypes.byref(c), heads, tokens, top) == 0
    assert q(None, 4, 20, 80) == 0
    assert q(ctypes.byref(A._cache(format=2)), 4, 20, 80) == 0


B, HK, H, D, PAGE, PAGES, CAP, M = 2, 2, 4, 128, 16, 9, 64, 7
F16, I32 = torch.float16, torch.int32
SHAPES = {
    "Q": ((M, H, D), F16), "k": ((PAGES, HK, PAGE, D), F16), "v": ((PAGES, HK, PAGE, D), F16),
    "table": ((B, CAP // PAGE), I32), "row_start": ((B + 1,), I32), "lengths": ((B,), I32),
    "mask": ((B, CAP), torch.bool), "out": ((M, H, D), F16), "workspace": ((1 << 20,), torch.uint8)}


def _python(t, **kw):
    rrs.prompt_attention(t["Q"], rrs.KVCache(t["k"], t["v"], t["table"]), t["row_start"],
                         t["lengths"], mask=t["mask"], out=t["out"], workspace=t["workspace"], **kw)


def _fake(**change):
    with FakeTensorMode():
        return {n: torch.empty(shape, **{**dict(dtype=dtype, device="cuda:0"),
                                         **change.get(n, {})})
                for n, (shape, dtype) in SHAPES.items()}


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
@pytest.mark.parametrize("device", ["cuda:1", "cpu"])
@pytest.mark.parametrize("name", [n for n in SHAPES if n != "Q"])
def test_another_device(name, device):
    with pytest.raises(ValueError, match="on cuda:0"):
        _python(_fake(**{name: dict(device=device)}))


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
def test_tensors():
    with pytest.raises(ValueError, match="GPU"):
        _python(_fake(Q=dict(device="cpu")))
    for name in ("Q", "v", "table", "row_start", "lengths", "mask", "out"):
        with pytest.raises(TypeError):
            _python(_fake(**{name: dict(dtype=torch.float64)}))
        with pytest.raises(ValueError):
            t = _fake()
            with FakeTensorMode():
                t[name] = torch.empty(tuple(x + 1 for x in SHAPES[name][0]), dtype=SHAPES[name][1],
                                      device="cuda:0")
            _python(t)
    with pytest.raises(TypeError):
        _python(_fake(), scale="1")
