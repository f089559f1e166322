"""RRS_DEBUG: a call that would write into a page of two rows is refused before anything is enqueued."""
import pytest
import torch

import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def debug_env(monkeypatch):
    monkeypatch.setenv("RRS_DEBUG", "1")


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _refused(call):
    with pytest.raises(rrs.RRSError) as e:
        call()
    assert "precondition" in str(e.value).lower(), str(e.value)


def _cache(table, fmt=rrs.KV_F16):
    cache = rrs.kv_cache(6, 1, 16, 64, _int(table), fmt)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).zero_()
    return cache


def _append(cache, seq, slot):
    M = len(seq)
    rrs.rope_kv_append(torch.ones((M, 3 * 64), dtype=torch.float16, device="cuda"),
                       _int([[0]] * M), rrs.rope_table(4, 64), cache, _int(seq), _int(slot), 1)


@pytest.mark.parametrize("fmt", [rrs.KV_F16, rrs.KV_FP8])
@pytest.mark.parametrize("table,seq,slot,good", [
    ([[0, 1], [2, 3]], [0, 1], [20, 20], True),
    ([[0, 1], [0, 3]], [0, 1], [20, 20], True),       # a shared full page
    ([[0, 1], [0, 1]], [0, 1], [20, 21], False),      # both write into the shared last page
    ([[0, 1], [1, 3]], [0, 1], [20, 20], False),      # one writes into what the other has filled
    ([[0, 1], [3, 0]], [0, 1], [3, 17], False),
    ([[0, 1], [3, 1]], [0, 1], [20, 3], True),        # the other's entry lies behind its token's
    ([[0, 1], [3, 1]], [0, 9], [20, 20], True),       # (not stored)
    ([[0, 1], [0, 1]], [0, 0, 1], [20, 21, -1], True),
    ([[0, 1], [-1, 3]], [0, 1], [20, 20], True),
    ([[5, 5], [2, 3]], [0, 1], [20, 20], True)])
def test_append(table, seq, slot, good, fmt):
    cache = _cache(table, fmt)
    if good:
        _append(cache, seq, slot)
    else:
        _refused(lambda: _append(cache, seq, slot))
        assert not cache.k.view(torch.uint8).any()


def test_append_after_fork():
    """A forked row that is given no room shares its last page; with room and its copy it does not."""
    cache = _cache([[0, 1], [2, 3], [-1, -1]])
    n, parent = _int([20, 5, 0]), _int([0, 1, 0])
    plan = rrs.kv_fork(cache.table, n, parent, _int([20, 5, 20]), 6, 16)
    _refused(lambda: _append(cache._replace(table=plan.table), [0, 2], [20, 20]))
    plan = rrs.kv_fork(cache.table, n, parent, _int([21, 6, 21]), 6, 16)
    rrs.kv_copy_pages(cache, plan.src, plan.dst, plan.count)
    _append(cache._replace(table=plan.table), [0, 1, 2], [20, 5, 20])


@pytest.mark.parametrize("table,lengths,good", [
    ([[0, 1], [2, 3]], [32, 20], True), ([[0, 1], [0, 3]], [32, 20], False),
    ([[0, 1], [2, 0]], [32, 16], True), ([[0, 1], [2, 0]], [32, 17], False),
    ([[0, 0], [2, 3]], [17, 1], False), ([[0, 0], [0, 0]], [0, 16], True)])
def test_evict(table, lengths, good):
    cache = _cache(table)
    w = torch.rand((2, 1, 32), device="cuda")
    pos = torch.arange(32, dtype=torch.int32, device="cuda").expand(2, 1, 32).contiguous()

    def call():
        rrs.kv_evict(cache, _int(lengths), w, pos, _int([30, 30]), 8)
    call() if good else _refused(call)
