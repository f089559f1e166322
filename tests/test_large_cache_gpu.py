"""Pools and batches past 2^32 bytes: the same calls on a small cache give the same bits. And refusals of overlapping
memory."""
import pytest
import torch

import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu

H, HK, D, P, N = 16, 8, 128, 256, 301


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("format,pages", [(rrs.KV_F16, 9000), (rrs.KV_INT4, 34000),
                                          (rrs.KV_FP8, 17000)])
def test_last_pages(format, pages):
    gen = torch.Generator().manual_seed(format)
    qkv = torch.randn((2 * N, (H + 2 * HK) * D), generator=gen).half().cuda()
    seq = _int([0] * N + [1] * N)
    slot = torch.arange(N, dtype=torch.int32).repeat(2).cuda()
    rope = rrs.rope_table(N, D)
    starts, n = _int([0, N, 2 * N]), _int([N, N])
    results = []
    for total, last in ((4, [2, 3]), (pages, [pages - 2, pages - 1])):
        cache = rrs.kv_cache(total, HK, P, D, _int([[0, 1], last]), format)
        q = rrs.rope_kv_append(qkv, slot.view(-1, 1), rope, cache, seq, slot, H)
        y, lse = rrs.prompt_attention(q, cache, starts, n, max_tokens=N, max_length=N,
                                      return_lse=True)
        one, one_lse = rrs.paged_attention(q[[N - 1, 2 * N - 1]], cache, n, max_length=N,
                                           return_lse=True)
        k, v = rrs.kv_read(cache, n, N)
        # The last sequence's pages swapped with pages that are free: the table follows.
        free = [total // 2 - 1, total // 2] if total > 4 else last
        if total > 4:
            assert cache.k.numel() * cache.k.element_size() > 1 << 32
            rrs.kv_copy_pages(cache, _int(last), _int(free))
            plan = rrs.kv_compact(_int([[0, 1], free]), n, total, P)
            rrs.kv_copy_pages(cache, plan.src, plan.dst, plan.count)
            cache = cache._replace(table=plan.table)
            assert plan.table.tolist() == [[0, 1], [2, 3]]
        again = rrs.prompt_attention(q, cache, starts, n, max_tokens=N, max_length=N)
        assert torch.equal(again, y)
        results.append((q, y, lse, one, one_lse, k, v))
    for x, z in zip(*results):
        assert torch.equal(x, z)


def test_many_query_bytes():
    """Queries and outputs of more than 2^32 bytes; a run longer than max_tokens is cut, its other rows stay."""
    heads, dim, M, n = 64, 256, 140001, 5
    gen = torch.Generator().manual_seed(0)
    cache = rrs.kv_cache(3, 2, 16, dim, _int([[0], [1], [2]]), rrs.KV_F16)
    cache.k.copy_(torch.randn(cache.k.shape, generator=gen))
    cache.v.copy_(torch.randn(cache.v.shape, generator=gen))
    few = torch.randn((3 * n, heads, dim), generator=gen).half().cuda()
    lengths = _int([16, 9, 5])
    want, want_lse = rrs.prompt_attention(few, cache, _int([0, n, 2 * n, 3 * n]), lengths,
                                          max_tokens=n, return_lse=True)
    Q = torch.zeros((M, heads, dim), dtype=torch.float16, device="cuda")
    places = torch.tensor([*range(n), *range(n, 2 * n), *range(M - n, M)])
    Q[places.cuda()] = few
    out = torch.full_like(Q, 7.0)
    y, lse = rrs.prompt_attention(Q, cache, _int([0, n, M - n, M]), lengths, max_tokens=n,
                                  return_lse=True, out=out)
    assert torch.equal(y[places.cuda()], want) and torch.equal(lse[places.cuda()], want_lse)
    assert bool((y[2 * n:M - n] == 7.0).all())


def test_overlaps():
    cache = rrs.kv_cache(4, 2, 16, 64, _int([[0, 1], [2, 3]]), rrs.KV_FP8)
    n, starts = _int([9, 3]), _int([0, 4, 6])
    Q = torch.randn((6, 4, 64), device="cuda").half()
    with pytest.raises(ValueError, match="out and Q must not overlap"):
        rrs.prompt_attention(Q, cache, starts, n, out=Q)
    with pytest.raises(ValueError, match="src"):
        rrs.kv_copy_pages(cache, cache.k.view(torch.int32).view(-1)[:2], _int([1, 2]))
    with pytest.raises(ValueError, match="count"):
        rrs.kv_copy_pages(cache, _int([0]), _int([1]), cache.v_scale.view(-1).view(torch.int32)[:1])
    with pytest.raises(ValueError, match="k and v must not overlap"):
        rrs.kv_copy_pages(cache._replace(v=cache.k), _int([0]), _int([1]))
    table, room = cache.table, _int([12, 20])
    plan = rrs.kv_fork(table, n, None, room, 4, 16)
    with pytest.raises(ValueError, match="table_out and table must not overlap"):
        rrs.kv_fork(table, n, None, room, 4, 16, out=(table, *plan[1:]))
    with pytest.raises(ValueError, match="src and dst must not overlap"):
        rrs.kv_fork(table, n, None, room, 4, 16, out=(*plan[:3], plan.src, plan.src, plan.count))
    c = rrs.kv_compact(table, n, 4, 16)
    with pytest.raises(ValueError, match="table_out and table must not overlap"):
        rrs.kv_compact(table, n, 4, 16, out=(table, *c[1:]))
