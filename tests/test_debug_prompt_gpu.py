"""RRS_DEBUG and prompt attention's rows: those of a sequence have to be finite, those of none (a padded batch) not."""
import math

import pytest
import torch

import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("starts", [[2, 4, 7], [0, 0, 3], [5, 9, 9], [4, 4, 4]])
def test_padded_rows(monkeypatch, starts):
    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    cache = rrs.kv_cache(4, 1, 16, 64, ints([[0, 1], [2, 3]]))
    cache.k.fill_(0.5), cache.v.fill_(0.25)
    M, n = 9, ints([20, 9])
    Q = torch.full((M, 2, 64), math.nan, dtype=torch.float16, device="cuda")
    Q[starts[0]:starts[2]] = 1.0

    def call():
        return rrs.prompt_attention(Q, cache, ints(starts), n, out=torch.full_like(Q, 3.0))
    want = call()
    monkeypatch.setenv("RRS_DEBUG", "1")
    assert torch.equal(call(), want)
    assert bool((want[starts[0]:starts[2]] == 0.25).all())
    for row in (starts[0], starts[2] - 1):
        if starts[0] == starts[2]:
            break
        Q[starts[0]:starts[2]] = 1.0
        Q[row, 1, 63] = math.inf
        with pytest.raises(rrs.RRSError, match="PRECONDITION"):
            call()
