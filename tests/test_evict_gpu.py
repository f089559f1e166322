"""kv_evict on the GPU: whole numbers and copies, so everything is compared exactly."""
import pytest
import torch

import paper_2409_20361_amd as rrs
from _kv_util import evict, make_cache

pytestmark = pytest.mark.gpu


def _check(cache, lengths, w, pos, keep_from, budget, max_length=None):
    B, hk = w.shape[:2]
    P = cache.k.shape[2]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    before = [t.clone() if t is not None else None for t in cache]
    w0, pos0 = w.clone(), pos.clone()
    kept, new, w2, pos2 = rrs.kv_evict(cache, i32(lengths), w, pos, i32(keep_from), budget,
                                       max_length)
    top = cache.capacity if max_length is None else max_length
    want = [None if t is None else t.clone() for t in before]
    for b in range(B):
        n = min(max(lengths[b], 0), top)
        m = min(n, budget)
        assert int(new[b]) == m
        for h in range(hk):
            at = evict(n, budget, w[b, h].cpu(), pos[b, h].cpu(), keep_from[b])
            assert kept[b, h].tolist() == at + [-1] * (budget - m), (b, h)
            src = torch.tensor(at, dtype=torch.long).cuda()
            assert torch.equal(w2[b, h, :m].view(torch.int32), w[b, h, src].view(torch.int32))
            assert not w2[b, h, m:].any()
            assert torch.equal(pos2[b, h, :m], pos[b, h, src])
            assert (pos2[b, h, m:] == -1).all()
            to = torch.arange(m).cuda()
            tp, sp = cache.table[b, to // P].long(), cache.table[b, src // P].long()
            for now, old in zip(want, before):
                if now is not None and now.dim() > 2:
                    now[tp, h, to % P] = old[sp, h, src % P]
    for now, exp in zip(cache, want):
        if now is not None:
            assert torch.equal(now, exp)
    assert torch.equal(w.view(torch.int32), w0.view(torch.int32)) and torch.equal(pos, pos0)


def _state(gen, B, hk, capacity, kind="random"):
    w = torch.exp(2 * torch.randn((B, hk, capacity), generator=gen)).cuda()
    if kind == "ties":
        w = torch.randint(0, 3, (B, hk, capacity), generator=gen).float().cuda()
    if kind == "equal":
        w = torch.full_like(w, 0.25)
    if kind == "odd":   # signed zeros, negative numbers, NaN of both signs
        pick = torch.tensor([0.0, -0.0, -1.0, 2.0, float("nan"), -float("nan"), 1e-40])
        w = pick[torch.randint(0, 7, (B, hk, capacity), generator=gen)].cuda()
    pos = torch.rand((B, hk, capacity), generator=gen).argsort(-1).int().cuda()
    return w, pos


@pytest.mark.parametrize("fmt", ["f16", "int4"])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (256, 32)])
def test_lengths_and_budgets(D, page, fmt):
    gen = torch.Generator().manual_seed(0)
    lengths = [0, 1, 5, 16, 63, 64, 65, 200]
    for budget in (1, 5, 64, 199, 200, 208):
        cache = make_cache(gen, len(lengths), 208, 2, D, page, fmt)
        w, pos = _state(gen, len(lengths), 2, cache.capacity)
        _check(cache, lengths, w, pos, [10 ** 6] * len(lengths), min(budget, cache.capacity))


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("n,budget", [(100, 37), (1025, 1024), (1024, 1023), (2049, 2048),
                                      (3000, 1), (5000, 2500), (9001, 4097)])
def test_kinds_of_weights(n, budget, kind):
    gen = torch.Generator().manual_seed(n)
    cache = make_cache(gen, 2, n, 3, 64, 16, "int4")
    w, pos = _state(gen, 2, 3, cache.capacity, kind)
    _check(cache, [n, n - 1], w, pos, [10 ** 6, n // 2], budget)


@pytest.mark.parametrize("keep_from", [0, 50, 95, 10 ** 6])
def test_protected(keep_from):
    """More protected slots than the budget, some, none."""
    gen = torch.Generator().manual_seed(keep_from)
    cache = make_cache(gen, 2, 100, 2, 128, 16, "f16")
    w, pos = _state(gen, 2, 2, cache.capacity, "ties")
    _check(cache, [100, 99], w, pos, [keep_from, 90], 40, 100)


@pytest.mark.parametrize("n,budget", [(33000, 8192), (40001, 40000), (140000, 100), (131072, 65536)])
def test_long(n, budget):
    gen = torch.Generator().manual_seed(n)
    cache = make_cache(gen, 1, n, 1, 64, 256, "int4")
    w, pos = _state(gen, 1, 1, cache.capacity, "random")
    w[..., ::5] = 0.0
    _check(cache, [n], w, pos, [n - 50], budget)


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("budget", [1, 8191, 8192, 8193, 20000, 24999])
def test_long_ragged(budget, kind):
    """Rows of several segments, of one, and of none, with ties across the segments' borders."""
    gen = torch.Generator().manual_seed(budget)
    lengths = [25000, 8192, 16385, 0, 24577]
    cache = make_cache(gen, len(lengths), 25000, 1, 64, 256, "int4")
    w, pos = _state(gen, len(lengths), 1, cache.capacity, kind)
    _check(cache, lengths, w, pos, [24900, 10 ** 6, 0, 0, 20000], budget, 25000)


@pytest.mark.parametrize("n,budget", [(16384, 9000), (16385, 9000), (4096, 4000), (4097, 64),
                                      (1024, 1020), (2000, 64), (2000, 65)])
def test_sides_of_the_kernels(n, budget):
    """Lengths and numbers of moves around those at which another kernel takes over."""
    gen = torch.Generator().manual_seed(n + budget)
    for fmt, D in (("f16", 256), ("int4", 64)):
        cache = make_cache(gen, 2, n, 2, D, 64, fmt)
        w, pos = _state(gen, 2, 2, cache.capacity, "ties")
        _check(cache, [n, n // 3], w, pos, [n - 9, 3], budget, n)


def test_bound_of_the_lengths():
    gen = torch.Generator().manual_seed(5)
    cache = make_cache(gen, 3, 300, 2, 64, 16, "f16")
    w, pos = _state(gen, 3, 2, cache.capacity)
    _check(cache, [300, -4, 120], w, pos, [290, 0, 0], 64, 150)


def test_streams_graph_and_repeats():
    """A call leaves its inputs alone, so it can be repeated: same bits, also from a graph."""
    gen = torch.Generator().manual_seed(6)
    cache = make_cache(gen, 2, 2000, 2, 128, 64, "f16")
    w, pos = _state(gen, 2, 2, cache.capacity, "ties")
    n = torch.tensor([2000, 1500], dtype=torch.int32).cuda()
    keep = torch.tensor([1990, 1490], dtype=torch.int32).cuda()
    want = [t.clone() for t in rrs.kv_evict(cache, n, w, pos, keep, 700)]
    k = cache.k.clone()
    out = tuple(torch.empty_like(t) for t in want)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        rrs.kv_evict(cache, n, w, pos, keep, 700, out=out)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(cache.k, k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rrs.kv_evict(cache, n, w, pos, keep, 700, out=out)
    for i in range(3):
        for t in out:
            t.fill_(7)
        w.copy_(torch.rand(w.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        again = rrs.kv_evict(cache, n, w, pos, keep, 700)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_refusals():
    gen = torch.Generator().manual_seed(7)
    cache = make_cache(gen, 2, 64, 2, 128, 16, "f16")
    w, pos = _state(gen, 2, 2, 64)
    n, keep = torch.tensor([64, 64], dtype=torch.int32).cuda(), torch.zeros(2).int().cuda()
    for budget in (0, 65):
        with pytest.raises(ValueError):
            rrs.kv_evict(cache, n, w, pos, keep, budget)
    with pytest.raises(rrs.RRSError, match="SHAPE"):
        rrs.kv_evict(cache, n, w, pos, keep, 8, max_length=65)
    with pytest.raises(TypeError):
        rrs.kv_evict(cache, n, w.double(), pos, keep, 8)
    with pytest.raises(ValueError):
        rrs.kv_evict(cache, n, w[:, :1], pos, keep, 8)
    long = make_cache(gen, 1, 20000, 1, 64, 256, "int4")
    w2, pos2 = _state(gen, 1, 1, long.capacity)
    need = rrs.kv_evict_workspace_bytes(long, 20000, 9)
    with pytest.raises(rrs.RRSError, match="WORKSPACE"):
        rrs.kv_evict(long, n[:1], w2, pos2, keep[:1], 9, 20000,
                     workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    out = rrs.kv_evict(cache, n, w, pos, keep, 8)
    with pytest.raises(ValueError):
        rrs.kv_evict(cache, n, w, pos, keep, 8, out=(out[0], out[1], w, out[3]))
