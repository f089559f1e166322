"""Prompt attention in the forms that its sizes choose: slots in many pieces, workgroups of eight waves."""
import math

import pytest
import torch

import _prompt_util as R
import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pieces(cache, heads, tokens, top, rows):
    """Pieces that the slots are cut into: the workspace holds D sums and three numbers for each and every row of
    the tiles of `rows` rows. Fails where the tiles are of another size, or the tokens few enough for another kernel."""
    B, hk, D = cache.table.shape[0], cache.k.shape[1], cache.k.shape[3]
    if cache.k.dtype == torch.uint8:
        D *= 2
    assert tokens * heads // hk > 128
    tiles = -(-tokens * heads // hk // rows)
    need = rrs.prompt_attention_workspace_bytes(cache, heads, tokens, top)
    unit = B * hk * tiles * rows * (4 * D + 12)
    assert need % unit == 0, (need, unit)
    return need // unit


@pytest.mark.parametrize("D,hk,L,fmt", [(128, 1, 5003, "fp8"), (256, 2, 3001, "int4"), (64, 1, 9001, "f16"),
                                        (128, 3, 2600, "int4"), (256, 1, 2000, "fp8")])
def test_join_by_groups(D, hk, L, fmt):
    """More than eight pieces, joined by several groups of threads; rows that see nothing, in some pieces or in all."""
    gen = torch.Generator().manual_seed(D + L)
    n, heads = 45, 3 * hk
    cache, plain = R.make_cache(gen, 1, L, hk, D, 64, fmt)
    assert _pieces(cache, heads, n, L, 128) > 8
    Q = torch.randn((n, heads, D), generator=gen).half().cuda()
    late = torch.ones((1, cache.capacity), dtype=torch.bool, device="cuda")
    late[0, :L - 20] = False
    early = torch.zeros_like(late)
    early[0, 5:90] = True
    for mask in (None, late, early):
        out, lse = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), max_length=L, mask=mask,
                                        return_lse=True)
        R.check(out, lse, R.attention(Q, plain, [(0, n)], [L], D ** -0.5, mask), [(0, n)])


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("L", [1500, 2300])
def test_eight_waves_in_pieces(L, mask, fmt):
    """Workgroups of eight waves whose slots are cut, with numbers that are not finite in slots that every row
    sees, that some do (on both sides of a tile's end), and that nobody does."""
    gen = torch.Generator().manual_seed(L)
    n, hk, heads, D, page = 260, 2, 8, 128, 32
    cache, plain = R.make_cache(gen, 1, L, hk, D, page, fmt)
    plain = rrs.KVCache(plain.k.clone(), plain.v.clone(), plain.table)
    assert _pieces(cache, heads, n, L, 256) == ((L - 1) // 64 + 1) // 4
    m = None
    if mask:
        m = (torch.rand((1, cache.capacity), generator=gen) < 0.7).cuda()
        m[0, 64 * (L // 64)], m[0, L - 130] = True, False
    slots = [5, 640, L - n - 1, L - n, L - n + 1, L - 130, 64 * (L // 64) - 1, 64 * (L // 64), L - 1]
    for i, t in enumerate(slots):
        p, at, h, d = int(cache.table[0, t // page]), t % page, i % hk, 3 + 11 * i
        what = (math.nan, math.inf, -math.inf)[i % 3]
        if fmt == "f16":
            cache.v[p, h, at, d] = what
            plain.v[p, h, at, d] = what
        elif fmt == "fp8":
            cache.v.view(torch.uint8)[p, h, at, d] = 127
            plain.v[p, h, at, d] = math.nan
        elif t >= L - n:   # (the scale of a whole row)
            cache.v_scale[p, h, at] = what
            plain.v[p, h, at] = math.nan
    Q = torch.randn((n, heads, D), generator=gen).half().cuda()
    out, lse = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), max_length=L, mask=m,
                                    return_lse=True)
    R.check(out, lse, R.attention(Q, plain, [(0, n)], [L], D ** -0.5, m), [(0, n)])
    # A key: NaN for the tokens that see it, for the others what was there.
    t = L - 30
    p, at = int(cache.table[0, t // page]), t % page
    if m is not None:
        m[0, t] = True
        out, lse = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), max_length=L, mask=m,
                                        return_lse=True)
    if fmt == "f16":
        cache.k[p, 0, at, 3] = math.inf
    elif fmt == "fp8":
        cache.k.view(torch.uint8)[p, 0, at, 3] = 255
    else:
        cache.k_scale[p, 0, at] = math.nan
    Q[:, :4, 3] = 1.0   # no infinity times 0
    before, before_lse = out, lse
    out, lse = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), max_length=L, mask=m,
                                    return_lse=True)
    assert bool(out[n - 30:, :4].isnan().all()) and bool(lse[n - 30:, :4].isnan().all())
    assert torch.equal(out[:, 4:].view(torch.int16), before[:, 4:].view(torch.int16))
    assert torch.equal(lse[:, 4:], before_lse[:, 4:])
    assert bool(lse[:n - 30].isfinite().all())


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("D,n,group,L", [(64, 70, 2, 300), (128, 70, 2, 300), (128, 260, 4, 700), (256, 70, 2, 200),
                                         (128, 7, 2, 300)])
def test_equal_values(D, n, group, L, fmt):
    """Slots that all hold the same value: the output is that value, whatever the weights and their rounding.

    With float16 weights p the output is sum p v / sum p. Both sums are float32 over no more than L products that are
    exact (11 bits each): with their rescaling each is off by at most 2 L 2^-24 relative, the quotient by
    less than 2^-12 for L <= 700, which rounds to the float16 number v. Two slots count, the second with 4 to 8 times
    the first's weight, in a later block: no weight but the first's is a power of two."""
    page, slot = 64, 100
    pages = -(-L // page)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    kind = {"f16": rrs.KV_F16, "int4": rrs.KV_INT4, "fp8": rrs.KV_FP8}[fmt]
    cache = rrs.kv_cache(pages, 1, page, D, table, kind)
    # Values of 2047 / 1024 (FP8: 15 / 8), whose half step is 2^-12 of them; keys of 0, but 1 at the slot.
    for pool in (cache.k, cache.v):
        pool.view(torch.uint8).zero_()
    if fmt == "f16":
        cache.v.fill_(2047 / 1024)
        cache.k[slot // page, 0, slot % page, 0] = 1.0
        v = 2047 / 1024
    elif fmt == "int4":
        cache.k_scale.fill_(1.0), cache.v_scale.fill_(2047 / 1024)
        cache.v.fill_(0x11)
        cache.k[slot // page, 0, slot % page, 0] = 1
        v = 2047 / 1024
    else:
        cache.k_scale.fill_(1.0), cache.v_scale.fill_(1.0)
        cache.v.view(torch.uint8).fill_(0x3F)
        cache.k.view(torch.uint8)[slot // page, 0, slot % page, 0] = 0x38
        v = 15 / 8
    mask = torch.zeros((1, cache.capacity), dtype=torch.bool, device="cuda")
    mask[0, 0] = mask[0, slot] = True
    scale = 0.125
    Q = torch.zeros((n, group, D), dtype=torch.float16, device="cuda")
    Q[:, :, 0] = torch.linspace(2.0, 2.98, n * group).view(n, group).cuda() * math.log(2) / scale
    for m in (mask, None):
        out, lse = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), max_length=L, scale=scale,
                                        mask=m, return_lse=True)
        assert bool((out == v).all()), (out.float() - v).abs().max().item()
    out = rrs.prompt_attention(Q, cache, _int([0, n]), _int([L]), scale=scale, mask=mask)
    assert bool((out == v).all())
