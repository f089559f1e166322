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
