"""RRS_DEBUG: what the FP8 append, prompt attention and the page calls need of device data is checked, and a call
that gets something else is refused before anything is enqueued; good calls pass."""
import pytest
import torch

import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


@pytest.fixture
def debug_env(monkeypatch):
    monkeypatch.setenv("RRS_DEBUG", "1")


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _refused(call):
    with pytest.raises(rrs.RRSError) as e:
        call()
    assert "precondition" in str(e.value).lower(), str(e.value)


def _cache(fmt=rrs.KV_FP8, table=((0, 1), (2, 3))):
    cache = rrs.kv_cache(4, 1, 16, 64, _int(table), fmt)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).zero_()
    return cache


def _append(seq, slot):
    cache = _cache()
    M = len(seq)
    rrs.rope_kv_append(torch.zeros((M, 3 * 64), dtype=torch.float16, device="cuda"),
                       _int([[0]] * M), rrs.rope_table(4, 64), cache, _int(seq), _int(slot), 1)


def test_runs(debug_env):
    _append([0, 0, 0, 1, -1, 1], [4, 5, 6, 15, 3, 16])
    _append([0, 9, 0], [3, 0, 16])
    for seq, slot in (([0, 0], [5, 4]), ([0, 0], [4, 6]), ([0, -1, 0], [4, 0, 5]),
                      ([1, 0, 1], [0, 0, 1]), ([0, 0], [7, 7])):
        _refused(lambda: _append(seq, slot))


@pytest.mark.parametrize("starts,lengths,tokens,good", [
    ([0, 3, 5], [10, 20], 3, True), ([0, 0, 0], [0, 1], 1, True), ([0, 3, 5], [10, 20], 2, False),
    ([0, 3, 2], [10, 20], 4, False), ([0, 3, 6], [10, 20], 4, False),
    ([-1, 3, 5], [10, 20], 4, False), ([0, 3, 5], [10, 33], 4, False)])
def test_prompt(debug_env, starts, lengths, tokens, good):
    Q = torch.zeros((5, 2, 64), dtype=torch.float16, device="cuda")

    def call():
        rrs.prompt_attention(Q, _cache(), _int(starts), _int(lengths), max_tokens=tokens)
    call() if good else _refused(call)


def test_prompt_table(debug_env):
    Q = torch.zeros((5, 2, 64), dtype=torch.float16, device="cuda")
    cache = _cache(table=((0, 9), (2, 3)))
    rrs.prompt_attention(Q, cache, _int([0, 5, 5]), _int([16, 7]))
    _refused(lambda: rrs.prompt_attention(Q, cache, _int([0, 5, 5]), _int([17, 7])))


def test_planners(debug_env):
    good, bad = _int([[0, 1], [2, 7]]), _int([[0, -1], [2, 7]])
    for n, table, fine in (([20, 16], good, True), ([16, 16], bad, True), ([20, 17], good, False),
                           ([20, 16], bad, False), ([33, 1], good, False), ([-1, 1], good, False)):
        for call in (lambda: rrs.kv_fork(table, _int(n), None, _int(n), 4, 16),
                     lambda: rrs.kv_compact(table, _int(n), 4, 16)):
            call() if fine else _refused(call)


def test_copies(debug_env):
    cache = _cache()
    for src, dst, count, fine in (
            ([0, 1], [2, 3], None, True), ([0, 1, 9], [2, 3, 9], 2, True), ([0, 0], [2, 3], None, True),
            ([0, 1, -1], [2, 3, -1], None, False), ([0, 1], [2, 2], None, False),
            ([0, 1], [1, 2], None, False), ([0, 1], [2, 3], 3, False), ([0, 4], [2, 3], None, False),
            ([0, 1], [2, 3], 0, True)):
        def call():
            rrs.kv_copy_pages(cache, _int(src), _int(dst), None if count is None else _int([count]))
        call() if fine else _refused(call)
