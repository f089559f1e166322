"""Host-only checks of the page calls: wrong arguments come back with the documented status, or are refused,
before any device is touched (no GPU needed; the pointers are never dereferenced)."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2409_20361_amd as rrs
import test_kv_abi as A

P, MIS = A.P, A.MIS


def _fork(**kw):
    a = dict(table=P, S=3, C=5, page=16, pages=9, lengths=P, parent=None, room=P, t2=P, n2=P, r2=P,
             src=P, dst=P, count=P, ws=P, bytes=1 << 40)
    a.update(kw)
    return rrs.lib().rrs_kv_fork(*a.values(), None)


def _compact(**kw):
    a = dict(table=P, S=3, C=5, page=16, pages=9, lengths=P, t2=P, src=P, dst=P, count=P, ws=P,
             bytes=1 << 40)
    a.update(kw)
    return rrs.lib().rrs_kv_compact(*a.values(), None)


def _copy(cache=None, **kw):
    a = dict(cache=ctypes.byref(cache or A._cache()), src=P, dst=P, n=4, count=None)
    a.update(kw)
    return rrs.lib().rrs_kv_copy_pages(*a.values(), None)


SHAPES = [dict(S=0), dict(S=1 << 23), dict(C=0), dict(C=(1 << 26) + 1), dict(page=8), dict(page=48),
          dict(page=512), dict(pages=0), dict(pages=(1 << 20) + 1)]


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, A.NULL) for n in ("table", "lengths", "room", "t2", "n2", "r2", "src", "dst",
                                    "count", "ws")],
    *[(kw, A.SHAPE) for kw in SHAPES],
    *[({n: MIS}, A.ALIGN) for n in ("table", "lengths", "parent", "room", "t2", "n2", "r2", "src",
                                    "dst", "count", "ws")],
    (dict(bytes=0), A.WS)])
def test_fork(kw, want):
    assert _fork(**kw) == want


@pytest.mark.parametrize("kw,want", [
    *[({n: None}, A.NULL) for n in ("table", "lengths", "t2", "src", "dst", "count", "ws")],
    *[(kw, A.SHAPE) for kw in SHAPES],
    *[({n: MIS}, A.ALIGN) for n in ("table", "lengths", "t2", "src", "dst", "count", "ws")],
    (dict(bytes=0), A.WS)])
def test_compact(kw, want):
    assert _compact(**kw) == want


def test_workspaces():
    for q, call in ((rrs.lib().rrs_kv_fork_workspace_bytes, _fork),
                    (rrs.lib().rrs_kv_compact_workspace_bytes, _compact)):
        need = q(3, 5, 16, 9)
        assert need > 0 and call(bytes=need - 1) == A.WS
        for kw in SHAPES:
            a = {**dict(S=3, C=5, page=16, pages=9), **kw}
            assert q(*a.values()) == 0


def test_copy():
    for kw, want in A.BAD_CACHES:
        assert _copy(A._cache(**kw)) == want, kw
    for kw, want in [(dict(src=None), A.NULL), (dict(dst=None), A.NULL), (dict(n=0), A.SHAPE),
                     (dict(src=MIS), A.ALIGN), (dict(dst=MIS), A.ALIGN), (dict(count=MIS), A.ALIGN)]:
        assert _copy(**kw) == want
    assert _copy(A._cache(kv_heads=1 << 20, sequences=1, head_dim=64)) == A.SHAPE   # 2^31 bytes a page


I32 = torch.int32
FORK = {"table": ((2, 5), I32), "lengths": ((2,), I32), "parent": ((2,), I32), "room": ((2,), I32),
        "table_out": ((2, 5), I32), "lengths_out": ((2,), I32), "room_out": ((2,), I32),
        "src": ((2,), I32), "dst": ((2,), I32), "count": ((2,), I32),
        "workspace": ((1 << 16,), torch.uint8)}
COMPACT = {**{k: FORK[k] for k in ("table", "lengths", "table_out", "count", "workspace")},
           "src": ((4,), I32), "dst": ((4,), I32)}
COPY = {"k": ((9, 2, 16, 64), torch.float16), "v": ((9, 2, 16, 64), torch.float16),
        "table": ((2, 5), I32), "src": ((4,), I32), "dst": ((4,), I32), "count": ((2,), I32)}


def _call_fork(t):
    rrs.kv_fork(t["table"], t["lengths"], t["parent"], t["room"], 9, 16,
                out=tuple(t[n] for n in ("table_out", "lengths_out", "room_out", "src", "dst",
                                         "count")), workspace=t["workspace"])


def _call_compact(t):
    rrs.kv_compact(t["table"], t["lengths"], 9, 16,
                   out=tuple(t[n] for n in ("table_out", "src", "dst", "count")),
                   workspace=t["workspace"])


def _call_copy(t):
    rrs.kv_copy_pages(rrs.KVCache(t["k"], t["v"], t["table"]), t["src"], t["dst"], t["count"])


CALLS = [(_call_fork, FORK, "table"), (_call_compact, COMPACT, "table"), (_call_copy, COPY, "k")]


def _fake(shapes, change=None):
    with FakeTensorMode():
        t = {n: torch.empty(shape, dtype=dtype, device="cuda:0")
             for n, (shape, dtype) in shapes.items()}
        if change:
            change(t)
    return t


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
@pytest.mark.parametrize("call,shapes,name", [(c, s, n) for c, s, lead in CALLS for n in s
                                              if n != lead])
@pytest.mark.parametrize("device", ["cuda:1", "cpu"])
def test_another_device(call, shapes, name, device):
    def change(t):
        t[name] = torch.empty(shapes[name][0], dtype=shapes[name][1], device=device)
    with pytest.raises(ValueError, match="on cuda:0"):
        call(_fake(shapes, change))


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
@pytest.mark.parametrize("call,shapes,name", [(c, s, n) for c, s, _ in CALLS for n in s
                                              if n not in ("workspace", "k", "v", "count")])
def test_types_and_shapes(call, shapes, name):
    def wrong_type(t):
        t[name] = torch.empty(shapes[name][0], dtype=torch.int64, device="cuda:0")

    def wrong_shape(t):
        t[name] = torch.empty(tuple(x + 1 for x in shapes[name][0]) + (2,), dtype=I32, device="cuda:0")
    with pytest.raises(TypeError):
        call(_fake(shapes, wrong_type))
    with pytest.raises(ValueError):
        call(_fake(shapes, wrong_shape))


def test_bad_out():
    t = _fake(FORK)
    with pytest.raises(TypeError, match="tuple"):
        rrs.kv_fork(t["table"], t["lengths"], None, t["room"], 9, 16, out=(t["table_out"],),
                    workspace=t["workspace"])
    with pytest.raises(ValueError, match="positive"):
        rrs.kv_compact(t["table"], t["lengths"], 0, 16)
    with pytest.raises(ValueError, match="GPU"):
        rrs.kv_fork(torch.zeros((2, 5), dtype=I32), t["lengths"], None, t["room"], 9, 16)
