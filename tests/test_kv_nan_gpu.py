"""Values that are not numbers stay visible through the cache's calls."""
import math

import pytest
import torch

import paper_2409_20361_amd as rrs
from _kv_util import make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_int4_append_keeps_rows_that_are_not_finite(D, bad):
    """A row with one such value and rows of nothing else are read back as NaN, and attention to
    them is NaN; the rows beside them are what they are without."""
    gen = torch.Generator().manual_seed(19)
    M, hk, page = 6, 2, 16
    cache = make_cache(gen, 1, M, hk, D, page, "int4")
    clean = [t.clone() for t in cache]
    rows = torch.randn((M, 3 * hk, D), generator=gen).half()
    want = rows.clone()
    # (token, head): of the keys hk + h, of the values 2 hk + h
    hit = {"k": [(1, 0), (4, 1)], "v": [(2, 1), (5, 0)]}
    for at, (one, all_) in ((hk, hit["k"]), (2 * hk, hit["v"])):
        rows[one[0], at + one[1], D - 3] = bad
        rows[all_[0], at + all_[1]] = bad
    idx = torch.arange(M, dtype=torch.int32).cuda()
    zero = torch.zeros_like(idx)
    n = torch.tensor([M], dtype=torch.int32).cuda()
    got = []
    for x, c in ((want, rrs.KVCache(*clean)), (rows, cache)):
        q = rrs.rope_kv_append(x.view(M, -1).cuda(), zero[:, None], rrs.rope_table(1, D), c, zero,
                               idx, hk)
        got.append((q, *rrs.kv_read(c, n, M)))
    assert torch.equal(got[0][0], got[1][0])
    for name, a, b in (("k", *[g[1] for g in got]), ("v", *[g[2] for g in got])):
        nan = torch.zeros((hk, M), dtype=torch.bool)
        for t, h in hit[name]:
            nan[h, t] = True
        assert torch.equal(b[0].isnan().all(-1).cpu(), nan), name
        assert torch.equal(b[0][~nan.cuda()], a[0][~nan.cuda()]), name
    out = rrs.paged_attention(want[M - 1:, :hk].contiguous().cuda(), cache, n, M)
    assert out.isnan().all()


@pytest.mark.parametrize("fmt", ["f16", "int4"])
@pytest.mark.parametrize("B,lengths", [(2, [40, 33]), (2, [9000, 7000]), (200, [40, 33])])
def test_not_a_number_reaches_the_weights(B, lengths, fmt):
    """A head whose softmax is NaN: the slots that take part get a NaN weight, no others do."""
    gen = torch.Generator().manual_seed(18)
    hk, D, page = 8, 128, 16
    lengths = [lengths[b % 2] for b in range(B)]
    top = max(lengths)
    cache = make_cache(gen, B, top, hk, D, page, fmt)
    Q = torch.randn((B, 2 * hk, D), generator=gen).half().cuda()
    mask = (torch.rand((B, cache.capacity), generator=gen) < 0.8).cuda()
    t = lengths[1] - 2   # of sequence 1, KV head 3
    mask[1, t] = True
    where = (cache.table[1, t // page].long(), 3, t % page)
    (cache.k if fmt == "f16" else cache.k_scale)[where] = math.nan
    w = torch.rand((B, hk, cache.capacity), generator=gen).cuda()
    w0 = w.clone()
    rrs.paged_attention(Q, cache, torch.tensor(lengths, dtype=torch.int32).cuda(), top, mask=mask,
                        weights=w)
    live = mask & (torch.arange(cache.capacity).cuda() < torch.tensor(lengths).cuda()[:, None])
    hit = torch.zeros((B, hk, 1), dtype=torch.bool, device="cuda")
    hit[1, 3] = True
    assert torch.equal(w.isnan(), live[:, None] & hit)
    dead = (~live)[:, None].expand_as(w)
    assert torch.equal(w[dead], w0[dead])
