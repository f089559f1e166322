"""The FP8 cache against plain forms: codes and scales bit for bit, attention in float64."""
import math

import pytest
import torch

import _fp8_util as F
import _kv_util as U
import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


def test_codes_and_units():
    """Every code in every scale reads as the float16 number that it stands for."""
    D, P = 64, 16
    scales = [2.0 ** e for e in range(-15, 9)]
    table = torch.arange(len(scales), dtype=torch.int32, device="cuda").view(1, -1)
    cache = rrs.kv_cache(len(scales), 1, P, D, table, rrs.KV_FP8)
    codes = torch.arange(256, dtype=torch.uint8).repeat(4).view(1, 1, P, D)
    for pool in (cache.k, cache.v):
        pool.view(torch.uint8).copy_(codes.expand(len(scales), 1, P, D))
    for s in (cache.k_scale, cache.v_scale):
        s.copy_(torch.tensor(scales).half().view(-1, 1, 1))
    n = len(scales) * P
    k, v = rrs.kv_read(cache, torch.tensor([n], dtype=torch.int32, device="cuda"))
    want = (F.E4M3[codes.long()] * torch.tensor(scales).double().view(-1, 1, 1, 1)).view(n, D)
    want16 = want.half()
    fits = want.abs() <= 61440
    assert bool((want16.double() == want)[fits].all())
    for got in (k, v):
        got = got[0, 0].cpu()
        assert torch.equal(got[fits], want16[fits])
        assert bool(got[want.isnan()].isnan().all())


def _append(gen, cache, qkv, seq, slot, heads, R, **kw):
    M = qkv.shape[0]
    pos = torch.randint(0, 50, (M, 1), generator=gen).int()
    rope = rrs.rope_table(50, R, device="cpu")
    q = rrs.rope_kv_append(qkv.cuda(), pos.cuda(), rope.cuda(), cache, seq.int().cuda(),
                           slot.int().cuda(), heads, **kw)
    # The same in float32, operation by operation.
    hk, D = cache.k.shape[1], cache.k.shape[3]
    x = qkv.float().view(M, heads + 2 * hk, D)
    c, s = rope[pos[:, 0].long(), None, :R // 2], rope[pos[:, 0].long(), None, R // 2:]
    y = x.clone()
    a, b = ((slice(0, R, 2), slice(1, R, 2)) if kw.get("interleaved") else
            (slice(0, R // 2), slice(R // 2, R)))
    qk = slice(0, heads + hk)
    y[:, qk, a] = x[:, qk, a] * c - x[:, qk, b] * s
    y[:, qk, b] = x[:, qk, b] * c + x[:, qk, a] * s
    y = y.half()
    return q, y[:, :heads], y[:, heads:heads + hk].double(), y[:, heads + hk:].double()


def _same(got, want):
    """Codes, where NaN may have either sign."""
    nan = (want & 127) == 127
    assert torch.equal(got[~nan], want[~nan]) and bool(((got & 127) == 127)[nan].all())


def _check(cache, before, rows, pools):
    """The cache after an append of rows [(seq, slot)] whose keys and values are pools."""
    P = cache.k.shape[2]
    want = [t.clone() for t in before]
    runs = []
    for m, (b, t) in enumerate(rows):
        if not (0 <= b < cache.table.shape[0] and 0 <= t < cache.capacity):
            continue
        if m and runs and runs[-1][2] == m and rows[m - 1] == (b, t - 1) and t % 16:
            runs[-1][2] += 1
        else:
            runs.append([m, m, m + 1])
    table = cache.table.cpu()
    for m, _, end in runs:
        b, t = rows[m]
        page, first = int(table[b, t // P]), t % 16
        for which, new in enumerate(pools):
            for h in range(new.shape[1]):
                blk = t % P // 16
                codes = want[which][page, h, blk * 16:blk * 16 + 16]
                want[2 + which][page, h, blk] = F.append(
                    codes, want[2 + which][page, h, blk], first, new[m:end, h])
    got = [cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale]
    for g, w in zip(got[2:], want[2:]):
        assert torch.equal(g.cpu(), w)
    for g, w in zip(got[:2], want[:2]):
        _same(g.cpu(), w)


def _bytes(cache):
    return [cache.k.view(torch.uint8).cpu(), cache.v.view(torch.uint8).cpu(),
            cache.k_scale.cpu(), cache.v_scale.cpu()]


@pytest.mark.parametrize("D,heads,hk,page,R,inter", [
    (128, 8, 2, 16, 128, False), (64, 5, 5, 32, 32, False), (256, 6, 1, 64, 64, True),
    (128, 33, 3, 128, 48, False), (64, 2, 2, 256, 64, True), (256, 3, 3, 16, 256, False)])
def test_append(D, heads, hk, page, R, inter):
    """Calls of one token, of some, of many; sequences interleaved with rows that are not stored."""
    gen = torch.Generator().manual_seed(D + heads)
    B, cap = 3, 128
    cache, _ = F.make_cache(gen, B, cap, hk, D, page)
    at = [0, 3, 17]
    for call, counts in enumerate([(5, 0, 1), (1, 1, 1), (1, 13, 30), (2, 1, 0), (37, 16, 15)]):
        rows = []
        for b in (2, 0, 1):
            rows += [(b, at[b] + i) for i in range(counts[b])] + [(-1, 0), (b, cap + 300)][:b]
            at[b] += counts[b]
        size = torch.exp2(3 * torch.randn((len(rows), 1), generator=gen))
        qkv = (size * torch.randn((len(rows), (heads + 2 * hk) * D), generator=gen)).half()
        seq, slot = (torch.tensor(x) for x in zip(*rows))
        before = _bytes(cache)
        q, q_want, k, v = _append(gen, cache, qkv, seq, slot, heads, R, interleaved=inter)
        assert torch.equal(q.cpu(), q_want)
        _check(cache, before, rows, (k, v))


@pytest.mark.parametrize("M,B,hk", [(768, 768, 3), (900, 5, 3), (1601, 97, 3), (600, 600, 1),
                                    (1100, 1100, 9), (1100, 300, 9), (2300, 900, 5)])
def test_append_many(M, B, hk):
    """Many windows of 16 rows, whose runs and heads are shared out among as many workgroups or fewer."""
    gen = torch.Generator().manual_seed(M)
    D, heads, page, cap = 64, 2 * hk, 32, 416 if B < 900 else 64
    cache, _ = F.make_cache(gen, B, cap, hk, D, page)
    cuts = torch.randperm(M - 1, generator=gen)[:B - 1].sort()[0] + 1
    counts = torch.diff(torch.cat([torch.tensor([0]), cuts, torch.tensor([M])])).tolist()
    start = torch.randint(0, 20, (B,), generator=gen).tolist()
    rows = [(b, start[b] + i) for b in range(B) for i in range(counts[b])]
    qkv = torch.randn((M, (heads + 2 * hk) * D), generator=gen).half()
    seq, slot = (torch.tensor(x) for x in zip(*rows))
    before = _bytes(cache)
    q, q_want, k, v = _append(gen, cache, qkv, seq, slot, heads, D)
    assert torch.equal(q.cpu(), q_want)
    _check(cache, before, rows, (k, v))


def test_append_bookkeeping():
    gen = torch.Generator().manual_seed(4)
    D, hk, heads, B, cap = 128, 2, 4, 2, 64
    cache, _ = F.make_cache(gen, B, cap, hk, D, 16)
    w = torch.ones((B, hk, cap), device="cuda")
    pos = torch.full((B, hk, cap), -1, dtype=torch.int32, device="cuda")
    seq, slot = torch.tensor([0, 0, 1, 9, 1]), torch.tensor([4, 5, 0, 1, 99])
    p = torch.tensor([[7], [8], [3], [4], [5]], dtype=torch.int32, device="cuda")
    rrs.rope_kv_append(torch.zeros((5, (heads + 2 * hk) * D), dtype=torch.float16, device="cuda"),
                       p, rrs.rope_table(50, D), cache, seq.int().cuda(), slot.int().cuda(), heads,
                       weights=w, slot_pos=pos)
    for t, stored, empty, values in ((w, 0.0, 1.0, [0, 0, 0]), (pos, None, -1, [7, 8, 3])):
        want = torch.full((B, hk, cap), empty, dtype=t.dtype)
        for (b, i), x in zip(((0, 4), (0, 5), (1, 0)), values):
            want[b, :, i] = x
        assert torch.equal(t.cpu(), want)


def test_not_finite():
    """NaN codes where a value is not finite; the block's other values and its scale are as without it."""
    gen = torch.Generator().manual_seed(5)
    D, hk, heads = 64, 1, 1
    cache, _ = F.make_cache(gen, 1, 32, hk, D, 32)
    rows = [(0, 16 + i) for i in range(4)]
    qkv = torch.randn((4, 3 * D), generator=gen)
    qkv[0, 2 * D + 3], qkv[1, 2 * D + 9], qkv[2, 2 * D:] = math.nan, math.inf, -math.inf
    qkv = qkv.half()
    before = _bytes(cache)
    seq, slot = (torch.tensor(x) for x in zip(*rows))
    _, _, k, v = _append(gen, cache, qkv, seq, slot, heads, D)
    _check(cache, before, rows, (k, v))
    _, got = rrs.kv_read(cache, torch.tensor([20], dtype=torch.int32, device="cuda"))
    bad = got[0, 0, 16:20].cpu().isnan()
    assert torch.equal(bad, ~qkv[:, 2 * D:].isfinite())


def test_largest_and_smallest():
    """float16's largest values stay finite; its smallest are kept exactly."""
    gen = torch.Generator().manual_seed(6)
    D = 64
    cache, _ = F.make_cache(gen, 1, 32, 1, D, 16)
    for first, size in ((0, 65504.0), (16, 2.0 ** -24)):
        qkv = torch.zeros((2, 3 * D))
        qkv[:, 2 * D:] = size * torch.randint(-8, 9, (2, D), generator=gen).clamp(
            *((-1, 1) if first == 0 else (-8, 8)))
        qkv[0, 2 * D] = size
        qkv = qkv.half()
        before = _bytes(cache)
        rows = [(0, first), (0, first + 1)]
        seq, slot = (torch.tensor(x) for x in zip(*rows))
        _, _, k, v = _append(gen, cache, qkv, seq, slot, 1, D)
        _check(cache, before, rows, (k, v))
        got = rrs.kv_read(cache, torch.tensor([18], dtype=torch.int32, device="cuda"))[1][0, 0]
        want = v[:, 0].clamp(-61440, 61440) if first == 0 else v[:, 0]
        assert torch.equal(got[first:first + 2].double().cpu(), want)


def test_scales_never_written():
    """A block without a scale so far (0, or any float16 that is none) takes the tokens' own."""
    gen = torch.Generator().manual_seed(7)
    D = 128
    for old in (0.0, math.inf, math.nan, -3.0, 40000.0):
        cache = rrs.kv_cache(2, 1, 16, D, torch.zeros((1, 1), dtype=torch.int32, device="cuda"),
                             rrs.KV_FP8)
        cache.k.view(torch.uint8).zero_()
        cache.v.view(torch.uint8).zero_()
        cache.k_scale.fill_(old), cache.v_scale.fill_(old)
        qkv = torch.randn((1, 3 * D), generator=gen).half()
        _append(gen, cache, qkv, torch.tensor([0]), torch.tensor([5]), 1, D)
        v = qkv[0, 2 * D:].double()
        e = F.exponent(float(v.abs().max()))
        assert float(cache.v_scale[0, 0, 0]) == 2.0 ** e
        got = cache.v.view(torch.uint8)[0, 0, 5].cpu()
        assert torch.equal(got, F.quantize(v, e))


def _compare(out, lse, w, w0, ref, B, H, lengths):
    for b in range(B):
        r = ref[b]
        if r is None:
            assert not out[b].any() and (lse is None or bool((lse[b] == -math.inf).all()))
            continue
        err = (out[b].double().cpu() - r["o"]).abs()
        assert bool((err <= r["tol"]).all()), (b, lengths[b], float((err - r["tol"]).max()))
        if lse is not None:
            assert float((lse[b].double().cpu() - r["lse"]).abs().max()) <= r["lse_tol"]
        if w is not None:
            n = lengths[b]
            gain = w[b, :, :n].double().cpu() - w0[b, :, :n].double()
            u = 2.0 ** -23 * (w0[b, :, :n].double() + r["w"])
            assert bool(((gain - r["w"]).abs() <= r["w_tol"] + u).all())


CASES = [
    # D, heads, hk, page, lengths, mask, weights
    (128, 4, 4, 64, [117], False, False), (128, 32, 8, 16, [1, 0, 64, 65, 300], False, True),
    (64, 10, 5, 32, [1, 2, 15, 16, 17, 33, 700], True, True),
    (256, 40, 1, 128, [512, 1, 31, 200], True, False), (256, 4, 2, 16, [65, 33], False, True),
    (128, 20, 1, 256, [4097, 3], False, True), (64, 64, 64, 16, [5, 64, 1, 30] * 16, False, False),
    (128, 64, 64, 32, [5, 33, 0, 30] * 16, True, False), (64, 3, 3, 64, [9001], False, False),
    (256, 32, 32, 16, [7, 1] * 40, False, False), (128, 8, 8, 64, [130] * 260, False, False),
]


@pytest.mark.parametrize("D,heads,hk,page,lengths,mask,weights", CASES)
def test_attention(D, heads, hk, page, lengths, mask, weights):
    gen = torch.Generator().manual_seed(D + heads + len(lengths))
    B, top = len(lengths), max(lengths)
    cache, plain = F.make_cache(gen, B, top + 20, hk, D, page)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    Q = torch.randn((B, heads, D), generator=gen).half().cuda()
    m = None
    if mask:
        m = (torch.rand((B, cache.capacity), generator=gen) < 0.6).cuda()
        m[-1] = False
    # Rows that take no part hold anything.
    slots = torch.arange(cache.capacity, device="cuda")
    dead = slots >= n[:, None] if m is None else (slots >= n[:, None]) | ~m
    for pool in (cache.k, cache.v):
        rows = pool.view(torch.uint8)
        for b in range(B):
            t = slots[dead[b]]
            rows[cache.table[b, t // page].long(), :, t % page] = 127
    # The scales of blocks none of whose slots take part, too.
    blocks = dead.view(B, -1, 16).all(-1)
    for b in range(B):
        j = torch.arange(blocks.shape[1], device="cuda")[blocks[b]]
        for s in (cache.k_scale, cache.v_scale):
            s[cache.table[b, j * 16 // page].long(), :, j * 16 % page // 16] = math.nan
    w = torch.rand((B, hk, cache.capacity), generator=gen).cuda() if weights else None
    w0 = w.cpu() if weights else None
    out, lse = rrs.paged_attention(Q, cache, n, max_length=max(top, 1), mask=m, weights=w,
                                   return_lse=True)
    ref = U.attention(Q, plain, lengths, D ** -0.5, m)
    _compare(out, lse, w, w0, ref, B, heads, lengths)
    if weights:
        for b in range(B):
            assert torch.equal(w[b, :, lengths[b]:].cpu(), w0[b, :, lengths[b]:])
    again = rrs.paged_attention(Q, cache, n, max_length=max(top, 1), mask=m)
    if not weights:
        assert torch.equal(again, out)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.5])
def test_attention_scale_and_spread(scale):
    """Blocks of very different scales, logits of any sign."""
    gen = torch.Generator().manual_seed(11)
    cache, plain = F.make_cache(gen, 2, 400, 2, 128, 32, spread=5.0)
    n = torch.tensor([400, 77], dtype=torch.int32, device="cuda")
    Q = torch.randn((2, 6, 128), generator=gen).half().cuda()
    out, lse = rrs.paged_attention(Q, cache, n, scale=scale, return_lse=True)
    _compare(out, lse, None, None, U.attention(Q, plain, [400, 77], scale), 2, 6, [400, 77])


def test_attention_nan():
    """A live slot's NaN shows in its heads, and nowhere else."""
    gen = torch.Generator().manual_seed(12)
    cache, _ = F.make_cache(gen, 2, 200, 2, 64, 16)
    n = torch.tensor([200, 150], dtype=torch.int32, device="cuda")
    Q = torch.randn((2, 4, 64), generator=gen).half().cuda()
    want = rrs.paged_attention(Q, cache, n)
    page = int(cache.table[0, 5])
    cache.v.view(torch.uint8)[page, 1, 3, 7] = 255
    got = rrs.paged_attention(Q, cache, n)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 2:, 7] = True
    assert bool(got[bad].isnan().all()) and torch.equal(got[~bad], want[~bad])
    cache.k.view(torch.uint8)[page, 0, 3, 7] = 127
    got, lse = rrs.paged_attention(Q, cache, n, return_lse=True)
    assert bool(got[0, :2].isnan().all()) and bool(lse[0, :2].isnan().all())
    assert torch.equal(got[1], want[1]) and bool(lse[0, 2:].isfinite().all())


def test_graph():
    """Append, attention and read-back in a graph, replayed with other tokens."""
    gen = torch.Generator().manual_seed(13)
    D, hk, heads, B = 128, 2, 8, 3
    caches = [F.make_cache(torch.Generator().manual_seed(13), B, 64, hk, D, 16)[0]
              for _ in range(2)]
    rope = rrs.rope_table(64, D)
    qkv = torch.zeros((B, (heads + 2 * hk) * D), dtype=torch.float16, device="cuda")
    seq = torch.arange(B, dtype=torch.int32, device="cuda")
    slot = torch.tensor([0, 15, 21], dtype=torch.int32, device="cuda")
    start = slot.clone()

    def step(cache, lengths):
        q = rrs.rope_kv_append(qkv, lengths.view(-1, 1), rope, cache, seq, lengths, heads)
        lengths += 1
        return rrs.paged_attention(q, cache, lengths, max_length=64), *rrs.kv_read(cache, lengths)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(caches[0], slot.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0], slot)
    slot.copy_(start)
    eager = start.clone()
    for t, s in zip(caches[0][:2] + caches[0][3:], caches[1][:2] + caches[1][3:]):
        t.view(torch.uint8).copy_(s.view(torch.uint8))
    for i in range(4):
        qkv.copy_(torch.randn(qkv.shape, generator=gen).half() * 2.0 ** i)
        graph.replay()
        for g, w in zip(got, step(caches[1], eager)):
            assert torch.equal(g, w)
        torch.cuda.synchronize()
