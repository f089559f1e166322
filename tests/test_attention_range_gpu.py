"""paged_attention where the weights of a softmax span many octaves (bounds: _kv_util.attention)."""
import math

import pytest
import torch

import paper_2409_20361_amd as rrs
from _kv_util import attention, make_cache, pack, quantize, values

pytestmark = pytest.mark.gpu

# One wave with the whole sequence, a workgroup with it, pieces joined.
WAYS = [(100, 16, 8, 100), (2, 4, 1, 256), (1, 4, 1, 3000)]


def _turned_to(gen, B, heads, hk, D):
    """Queries that are close to one direction per KV head, and the directions (B, hk, D)."""
    base = torch.randn((B, hk, D), generator=gen)
    noise = torch.randn((B, hk, heads // hk, D), generator=gen)
    return (base[:, :, None] + 0.05 * noise).view(B, heads, D).half(), base


@pytest.mark.parametrize("e,octaves", [(10, 30), (13, 40)])
@pytest.mark.parametrize("B,heads,hk,n", WAYS)
def test_int4_large_scale_of_a_slot_without_weight(B, heads, hk, n, e, octaves):
    """A live slot whose values are large and whose weight is next to nothing takes no bits from
    the others."""
    gen = torch.Generator().manual_seed(16)
    D, page, t = 128, 16, 5
    cache = make_cache(gen, B, n, hk, D, page, "int4")
    cache.v_scale.fill_(2.0 ** -6)
    Q, base = _turned_to(gen, B, heads, hk, D)
    at = (cache.table[:, t // page].long(), slice(None), t % page)
    cache.k[at] = pack(-7 * base.sign().long()).cuda()
    logit = 7 * base.abs().sum(-1) * D ** -0.5   # of a key scale of 1
    cache.k_scale[at] = (octaves * math.log(2.0) / logit).half().cuda()
    cache.v_scale[at] = 2.0 ** e
    lengths = [n] * B
    out = rrs.paged_attention(Q.cuda(), cache, torch.tensor(lengths, dtype=torch.int32).cuda(), n)
    for b, r in enumerate(attention(Q.cuda(), cache, lengths, D ** -0.5)):
        assert ((out[b].double().cpu() - r["o"]).abs() <= r["tol"]).all(), b


OCTAVES = [16, 22, 25, 26, 30]   # of the other slots below the sink


def _sink(B, heads, hk, n, octaves, fmt):
    """A slot that takes nearly all of the weight and holds zeros: the others make the output.

    Beside the common bound that of a subnormal weight: the products take weights as float16
    in units that leave 2^12 or more for the largest one so far (INT4: 2^11 for the largest product), so
    that half a subnormal step is 2^-25 2^-12 of it."""
    gen = torch.Generator().manual_seed(17)
    D, page, t = 128, 16, 0
    Q, base = _turned_to(gen, B, heads, hk, D)
    cache = make_cache(gen, B, n, hk, D, page, "f16")
    cache.k.mul_(0.01)
    cache.v.copy_((1000.0 * (1.0 + 0.1 * torch.randn(cache.v.shape, generator=gen))).half())
    at = (cache.table[:, t // page].long(), slice(None), t % page)
    q2 = (base * base).sum(-1, keepdim=True) * D ** -0.5
    cache.k[at] = (base * (octaves * math.log(2.0) / q2)).half().cuda()
    cache.v[at] = 0.0
    if fmt == "int4":
        k, v = (quantize(x.double().cpu()) for x in cache[:2])
        cache = rrs.KVCache(pack(k[0]).cuda(), pack(v[0]).cuda(), cache.table, k[1].cuda(),
                            v[1].cuda())
    lengths = [n] * B
    out = rrs.paged_attention(Q.cuda(), cache, torch.tensor(lengths, dtype=torch.int32).cuda(), n)
    for b, r in enumerate(attention(Q.cuda(), cache, lengths, D ** -0.5)):
        rest = 2.0 ** -37 * values(cache, b, n)[1].abs().sum(1)   # the sink's weight is below 1
        tol = r["tol"] + rest.repeat_interleave(heads // hk, 0)
        assert ((out[b].double().cpu() - r["o"]).abs() <= tol).all(), b


@pytest.mark.parametrize("octaves", OCTAVES)
@pytest.mark.parametrize("B,heads,hk,n", WAYS)
def test_int4_sink_without_a_value(B, heads, hk, n, octaves):
    _sink(B, heads, hk, n, octaves, "int4")


@pytest.mark.parametrize("octaves", OCTAVES)
@pytest.mark.parametrize("B,heads,hk,n", WAYS)
def test_f16_sink_without_a_value(B, heads, hk, n, octaves):
    _sink(B, heads, hk, n, octaves, "f16")
