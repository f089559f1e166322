"""kv_evict refuses outputs that share memory with what it reads, and only those."""
import pytest
import torch

import paper_2409_20361_amd as rrs
from _kv_util import make_cache

pytestmark = pytest.mark.gpu

B, HK, CAP = 4, 2, 64
NAMES = ["kept", "new_lengths", "weights_out", "pos_out", "lengths", "weights", "slot_pos",
         "keep_from"]


def _state():
    gen = torch.Generator().manual_seed(20)
    cache = make_cache(gen, B, CAP, HK, 64, 16, "int4")
    shape = (B, HK, CAP)
    t = {"kept": torch.empty(shape, dtype=torch.int32), "new_lengths": torch.empty(B).int(),
         "weights_out": torch.empty(shape), "pos_out": torch.empty(shape, dtype=torch.int32),
         "lengths": torch.tensor([64, 30, 64, 7]).int(), "weights": torch.rand(shape, generator=gen),
         "slot_pos": torch.rand(shape, generator=gen).argsort(-1).int(),
         "keep_from": torch.tensor([60, 0, 10, 0]).int()}
    return cache, {n: x.cuda() for n, x in t.items()}


def _call(cache, t, workspace=None):
    return rrs.kv_evict(cache, t["lengths"], t["weights"], t["slot_pos"], t["keep_from"],
                        t["kept"].shape[2], workspace=workspace,
                        out=tuple(t[n] for n in NAMES[:4]))


PAIRS = [(a, b) for i, a in enumerate(NAMES[:4]) for b in NAMES[i + 1:]]


@pytest.mark.parametrize("a,b", PAIRS)
def test_shared(a, b):
    """The two begin at the same place, or the one at the other's last 16 bytes."""
    for last in (False, True):
        cache, t = _state()
        x, y = t[a], t[b]
        room = torch.empty(x.nbytes + y.nbytes, dtype=torch.uint8, device="cuda")
        at = y.nbytes - 16 if last else 0
        y2 = room[:y.nbytes].view(y.dtype).view(y.shape)
        y2.copy_(y)
        t[b] = y2
        t[a] = room[at:at + x.nbytes].view(x.dtype).view(x.shape)
        want = {n: v.clone() for n, v in t.items()}
        k = cache.k.clone()
        with pytest.raises(ValueError, match=f"{a} and {b} must not overlap"):
            _call(cache, t)
        torch.cuda.synchronize()
        assert torch.equal(cache.k, k)
        for n in NAMES[4:]:
            assert torch.equal(t[n], want[n])


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale", "table"])
def test_shared_with_the_cache(name):
    cache, t = _state()
    room = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    x = getattr(cache, name)
    y = room[:x.nbytes].view(x.dtype).view(x.shape)
    y.copy_(x)
    cache = cache._replace(**{name: y})
    t["new_lengths"] = room[16:16 + 4 * B].view(torch.int32)
    with pytest.raises(ValueError, match=f"new_lengths and {name} must not overlap"):
        _call(cache, t)


def test_workspace():
    """It shares memory with an input, or would if the call needed one."""
    cache, t = _state()
    assert rrs.kv_evict_workspace_bytes(cache, CAP, CAP) == 0
    _call(cache, t, t["weights"].view(torch.uint8))
    gen = torch.Generator().manual_seed(21)
    cache = make_cache(gen, 1, 17000, 1, 64, 256, "int4")
    shape = (1, 1, cache.capacity)
    room = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    need = rrs.kv_evict_workspace_bytes(cache, 17000, 100)
    up = (need + 15) // 16 * 16   # arrays begin at multiples of 16 bytes
    assert 0 < up <= room.nbytes - 4 * cache.capacity
    n = torch.tensor([17000], dtype=torch.int32).cuda()
    pos = torch.zeros(shape, dtype=torch.int32, device="cuda")
    w = room[up - 16:up - 16 + 4 * cache.capacity].view(torch.float32).view(shape)
    with pytest.raises(ValueError, match="workspace and weights must not overlap"):
        rrs.kv_evict(cache, n, w, pos, n, 100, 17000, workspace=room)
    w = room[up:up + 4 * cache.capacity].view(torch.float32).view(shape)
    rrs.kv_evict(cache, n, w, pos, n, 100, 17000, workspace=room)
    torch.cuda.synchronize()


def test_neighbours_are_no_overlap():
    """All arguments side by side in one allocation: as with memory of their own."""
    cache, t = _state()
    other = rrs.KVCache(*(x.clone() for x in cache))
    t2 = {n: x.clone() for n, x in t.items()}
    room = torch.empty(sum(x.nbytes for x in t.values()), dtype=torch.uint8, device="cuda")
    at = 0
    for n, x in t.items():
        y = room[at:at + x.nbytes].view(x.dtype).view(x.shape)
        y.copy_(x)
        t[n], at = y, at + x.nbytes
    for x, y in zip(_call(cache, t), _call(other, t2)):
        assert torch.equal(x, y)
    assert all(torch.equal(x, y) for x, y in zip(cache, other))
