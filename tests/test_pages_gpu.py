"""Page planners against lists, page copies byte for byte."""
import random

import pytest
import torch

import _pages_util as G
import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _table(r, S, C, pages, P, share=0.5, dense=1.0):
    """A random table with lengths; rows may share their first pages. Each page is in a row once."""
    lengths = [r.choice([0, 1, C * P, r.randint(0, C * P), r.randint(0, C * P) // P * P])
               for _ in range(S)]
    free = list(range(pages))
    r.shuffle(free)
    rows = []
    for b in range(S):
        need = -(-lengths[b] // P)
        row = []
        if rows and r.random() < share:
            p = r.randrange(b)
            k = r.randint(0, min(need, -(-lengths[p] // P)))
            row = rows[p][:k]
        while len(row) < need and free:
            row.append(free.pop())
        lengths[b] = min(lengths[b], len(row) * P)
        rows.append(row + [-7] * (C - len(row)))
    return rows, lengths


def _check_fork(rows, lengths, parent, room, pages, P):
    want = G.fork(rows, lengths, parent, room, pages, P)
    got = rrs.kv_fork(_int(rows), _int(lengths), None if parent is None else _int(parent),
                      _int(room), pages, P)
    for name, x in want.items():
        assert getattr(got, name).tolist() == x, name
    return want


SIZES = [  # sequences, entries, page size, pages
    (1, 1, 16, 1), (1, 1, 16, 2), (3, 5, 16, 9), (8, 7, 32, 60), (70, 4, 16, 130), (1100, 3, 64, 2000),
    (2, 700, 16, 900), (33, 9, 256, 65), (2500, 9, 16, 12000), (40, 900, 16, 20000), (5, 60, 16, 70001),
    (3, 4, 128, 1 << 20), (6000, 7, 16, 9000)]


@pytest.mark.parametrize("S,C,P,pages", SIZES)
def test_fork(S, C, P, pages):
    r = random.Random(S + C + pages)
    for trial in range(4 if S * C < 2000 else 2):
        rows, lengths = _table(r, S, C, pages, P)
        parent = [r.choice([b, r.randrange(S), r.randrange(S), -1, S]) for b in range(S)]
        if trial == 0:
            parent = None
        grow = [1, 1, 5 * P, C * P][trial]
        room = [(lengths[b if parent is None else parent[b]]
                 if parent is None or 0 <= parent[b] < S else 0) + r.choice([0, grow, -grow])
                for b in range(S)]
        _check_fork(rows, lengths, parent, room, pages, P)


@pytest.mark.parametrize("S,C,P", [(40, 6, 16), (3000, 12, 16)])
def test_fork_not_enough(S, C, P):
    """A pool that runs out: from nothing left to one page less than needed."""
    r = random.Random(S)
    rows, lengths = _table(r, S, C, 10 ** 6, P)
    used = sorted({p for row, n in zip(rows, lengths) for p in row[:-(-n // P)]})
    to = {p: i for i, p in enumerate(used)}
    rows = [[to.get(p, -1) for p in row] for row in rows]
    parent = [r.choice([b, r.randrange(S)]) for b in range(S)]
    room = [lengths[p] + r.choice([0, 1, 1, 3 * P]) for p in parent]
    full = G.fork(rows, lengths, parent, room, 10 ** 6, P)
    took = 10 ** 6 - full["count"][1] - len({
        p for q, n in zip(parent, full["lengths"]) for p in rows[q][:-(-n // P)]})
    for extra in (0, 1, took // 2, took - 1, took):
        kept = {p for q, n in zip(parent, full["lengths"]) for p in rows[q][:-(-n // P)]}
        pages = max(max(kept) + 1, len(kept) + extra)
        _check_fork(rows, lengths, parent, room, pages, P)


def test_fork_last_pages():
    """Who copies a shared, partly filled page: all writers but the first if all that keep it write."""
    P, table = 16, [[3, 4, -1], [5, -1, -1], [0, 1, 2]]
    n = [20, 16, 40]
    for parent, room, src in [
            ([0, 0, 0], [21, 21, 21], [4, 4]), ([0, 0, 0], [20, 21, 21], [4, 4]),
            ([0, 0, 0], [21, 21, 20], [4, 4]), ([0, 0, 0], [20, 20, 20], []),
            ([0, 0, 0], [16, 21, 10], []), ([1, 1, 1], [17, 17, 17], []),
            ([0, 0, -1], [18, 40, 0], [4]), ([2, 2, 0], [48, 41, 99], [2])]:
        want = _check_fork(table, n, parent, room, 12, P)
        assert [p for p in want["src"] if p >= 0] == src


def test_fork_bad_numbers():
    """Lengths, rooms, parents and entries that are out of range stay harmless."""
    table = [[0, 99, 2], [-5, 1, 3], [2, 2, -1]]
    for n, parent, room in [([100, -3, 40], [0, 1, 2], [1000, 1000, 1000]),
                            ([20, 40, 17], [1, 0, 2 ** 31 - 1], [21, -5, 3]),
                            ([2 ** 31 - 1] * 3, None, [2 ** 31 - 1] * 3),
                            ([33, 33, 33], [1, 1, 0], [34, 34, 20])]:
        _check_fork(table, n, parent, room, 6, 16)


@pytest.mark.parametrize("S,C,P,pages", SIZES)
def test_compact(S, C, P, pages):
    r = random.Random(7 * S + C + pages)
    for trial in range(3):
        rows, lengths = _table(r, S, C, pages, P)
        if trial == 2:
            lengths = [n * r.randint(0, 1) for n in lengths]
            if S > 1 and rows[0]:
                rows[0][0] = pages + 5
        want = G.compact(rows, lengths, pages, P)
        got = rrs.kv_compact(_int(rows), _int(lengths), pages, P)
        for name, x in want.items():
            assert getattr(got, name).tolist() == x, name


def _random_cache(gen, pages, hk, P, D, fmt, table):
    cache = rrs.kv_cache(pages, hk, P, D, table, fmt)
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if t is not None:
            b = t.view(torch.uint8)
            b.copy_(torch.randint(0, 256, b.shape, generator=gen, dtype=torch.uint8))
    return cache


@pytest.mark.parametrize("fmt", [rrs.KV_F16, rrs.KV_INT4, rrs.KV_FP8])
@pytest.mark.parametrize("hk,P,D", [(1, 16, 64), (3, 32, 128), (8, 64, 128), (5, 256, 256)])
def test_copy(fmt, hk, P, D):
    gen = torch.Generator().manual_seed(hk + P + fmt)
    pages = 61
    cache = _random_cache(gen, pages, hk, P, D, fmt, _int([[0]]))
    perm = torch.randperm(pages, generator=gen).int()
    src, dst = perm[:20].clone(), perm[20:40].clone()
    src[3], dst[7], src[9], dst[11] = -1, pages, 2 ** 31 - 1, -2 ** 31
    for count in (None, 0, 1, 13, 20, 99, -1):
        want = []
        for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            if t is not None:
                w = t.view(torch.uint8).cpu().clone()
                n = 20 if count is None else min(max(count, 0), 20)
                ok = [i for i in range(n) if 0 <= src[i] < pages and 0 <= dst[i] < pages]
                w[dst[ok].long()] = w[src[ok].long()]
                want.append((t, w))
        c = None if count is None else _int([count, 5])
        assert rrs.kv_copy_pages(cache, src.cuda(), dst.cuda(), c) is None
        for t, w in want:
            assert torch.equal(t.view(torch.uint8).cpu(), w)
    assert rrs.kv_copy_pages(cache, src[:0].cuda(), dst[:0].cuda()) is None


def test_copy_many():
    """More pieces than workgroups."""
    gen = torch.Generator().manual_seed(3)
    pages = 6000
    cache = _random_cache(gen, pages, 2, 16, 64, rrs.KV_F16, _int([[0]]))
    perm = torch.randperm(pages, generator=gen).cuda().int()
    src, dst = perm[:2900], perm[2900:5800].contiguous()
    want = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
    for w in want:
        w[dst.long()] = w[src.long()]
    rrs.kv_copy_pages(cache, src, dst)
    for t, w in zip(cache, want):
        assert torch.equal(t.view(torch.uint8), w)


def test_copy_past_2_to_31():
    """A pool of more than 2^31 bytes."""
    pages, hk, P, D = 9000, 8, 128, 128
    cache = rrs.kv_cache(pages, hk, P, D, _int([[0]]), rrs.KV_F16)
    cache.k[[1, 8999]] = 1.0
    cache.k[8999] = torch.randn((hk, P, D), device="cuda").half()
    cache.v[0] = torch.randn((hk, P, D), device="cuda").half()
    rrs.kv_copy_pages(cache, _int([8999, 0]), _int([1, 8998]))
    assert torch.equal(cache.k[1], cache.k[8999]) and torch.equal(cache.v[0], cache.v[8998])


def test_out_and_workspace():
    rows, lengths = [[3, 1], [2, 0]], [20, 32]
    args = (_int(rows), _int(lengths), _int([0, 0]), _int([21, 30]), 6, 16)
    first = rrs.kv_fork(*args)
    out = tuple(torch.empty_like(t) for t in first)
    ws = torch.empty(rrs.kv_fork_workspace_bytes(2, 2, 16, 6), dtype=torch.uint8, device="cuda")
    for _ in range(3):   # the workspace's contents do not matter
        got = rrs.kv_fork(*args, out=out, workspace=ws)
        assert all(x.data_ptr() == y.data_ptr() for x, y in zip(got, out))
        assert all(torch.equal(x, y) for x, y in zip(got, first))
        ws.random_()
    c = rrs.kv_compact(args[0], args[1], 6, 16)
    out = tuple(torch.empty_like(t) for t in c)
    ws = torch.empty(rrs.kv_compact_workspace_bytes(2, 2, 16, 6), dtype=torch.uint8, device="cuda")
    got = rrs.kv_compact(args[0], args[1], 6, 16, out=out, workspace=ws)
    assert all(torch.equal(x, y) for x, y in zip(got, c))


@pytest.mark.parametrize("fmt", [rrs.KV_F16, rrs.KV_INT4, rrs.KV_FP8])
@pytest.mark.parametrize("large", [False, True])
def test_graph(fmt, large):
    """Fork and compact with their copies in one graph, replayed over other tables."""
    gen = torch.Generator().manual_seed(fmt)
    S, C, P = (6, 7000, 16) if large else (6, 5, 16)
    pages = 60
    r = random.Random(2)
    cache = _random_cache(gen, pages, 2, P, 64, fmt, _int([[0] * C] * S))
    twin = rrs.KVCache(*(t.clone() if t is not None else None for t in cache))
    lengths, parent, room = (_int([0] * S) for _ in range(3))

    def step(c):
        f = rrs.kv_fork(cache.table, lengths, parent, room, pages, P)
        rrs.kv_copy_pages(c, f.src, f.dst, f.count)
        m = rrs.kv_compact(f.table, f.room, pages, P)
        rrs.kv_copy_pages(c, m.src, m.dst, m.count)
        return (*f, *m)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(twin)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache)
    for _ in range(4):
        rows, n = _table(r, S, 5, pages, P)
        p = [r.randrange(S) for _ in range(S)]
        cache.table[:, :5] = _int(rows)
        lengths.copy_(_int(n)), parent.copy_(_int(p))
        room.copy_(_int([min(n[q] + 20, 80) for q in p]))
        graph.replay()
        want = step(twin)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        for x, y in zip(cache, twin):
            if x is not None and x.dtype != torch.int32:
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        torch.cuda.synchronize()
