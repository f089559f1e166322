"""Prompt attention against its plain form in float64."""
import math

import pytest
import torch

import _prompt_util as R
import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(counts, before=0):
    s = [before]
    for n in counts:
        s.append(s[-1] + n)
    return s, list(zip(s, counts))


def _fill_dead(cache, n, mask, fmt):
    """Slots past the lengths and under the mask hold NaN (INT4: under a scale that is NaN)."""
    P = cache.k.shape[2]
    slots = torch.arange(cache.capacity, device="cuda")
    dead = slots >= n[:, None] if mask is None else (slots >= n[:, None]) | ~mask
    for b in range(len(n)):
        t = slots[dead[b]]
        page, at = cache.table[b, t // P].long(), t % P
        for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            if fmt == "f16":
                pool[page, :, at] = math.nan
            elif fmt == "int4":
                scale[page, :, at] = math.nan
            else:
                pool.view(torch.uint8)[page, :, at] = 127
        if fmt == "fp8":   # scales of blocks none of whose slots take part
            j = slots[::16][dead[b].view(-1, 16).all(-1)]
            for scale in (cache.k_scale, cache.v_scale):
                scale[cache.table[b, j // P].long(), :, j % P // 16] = math.nan


CASES = [
    # D, heads, hk, page, [(new, length)], mask
    (128, 8, 2, 64, [(5, 5)], False), (128, 8, 8, 16, [(1, 1), (130, 130), (0, 40), (7, 300)], False),
    (64, 20, 5, 32, [(7, 1500), (1, 2), (3, 17), (64, 64)], False),
    (64, 4, 1, 16, [(33, 50), (0, 0), (1, 9)], True), (256, 40, 1, 128, [(3, 700), (17, 17)], True),
    (256, 4, 2, 64, [(200, 260)], False), (128, 4, 4, 256, [(300, 300), (1, 500)], True),
    (128, 32, 8, 32, [(9, 2100)], False), (64, 3, 3, 16, [(2, 2)] * 30, False),
    (128, 16, 16, 16, [(20, 33)] * 5, True), (128, 9, 3, 64, [(150, 1000)], False),
    (256, 8, 8, 16, [(31, 31), (70, 200)], False), (64, 64, 1, 64, [(65, 129)], False),
]


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("D,heads,hk,page,seqs,mask", CASES)
def test_attention(D, heads, hk, page, seqs, mask, fmt):
    gen = torch.Generator().manual_seed(D + heads + len(seqs))
    counts, lengths = zip(*seqs)
    B, top = len(seqs), max(max(lengths), 1)
    cache, plain = R.make_cache(gen, B, top + 20, hk, D, page, fmt)
    if fmt == "f16":
        plain = rrs.KVCache(cache.k.clone(), cache.v.clone(), cache.table)
    starts, rows = _starts(counts, 2)
    M = starts[-1] + 3
    Q = torch.randn((M, heads, D), generator=gen).half().cuda()
    n = _int(lengths)
    m = None
    if mask:
        m = (torch.rand((B, cache.capacity), generator=gen) < 0.6).cuda()
        m[:, 0] = False
        m[-1] = False
    _fill_dead(cache, n, m, fmt)
    out = torch.full_like(Q, 7.0)
    got, lse = rrs.prompt_attention(Q, cache, _int(starts), n, max_tokens=max(max(counts), 1),
                                    max_length=top, mask=m, return_lse=True, out=out)
    assert got.data_ptr() == out.data_ptr()
    assert bool((out[:2] == 7.0).all()) and bool((out[starts[-1]:] == 7.0).all())
    R.check(out, lse, R.attention(Q, plain, rows, lengths, D ** -0.5, m), rows)
    # Loose bounds (other pieces, other tiles) and no lse; the first call again, bit for bit.
    loose = rrs.prompt_attention(Q, cache, _int(starts), n, mask=m)
    R.check(loose, lse, R.attention(Q, plain, rows, lengths, D ** -0.5, m), rows)
    again = rrs.prompt_attention(Q, cache, _int(starts), n, max_tokens=max(max(counts), 1),
                                 max_length=top, mask=m)
    at = slice(2, starts[-1])
    assert torch.equal(again[at], out[at])


FEW = [
    # D, heads, hk, page, [(new, length)], mask: up to 16 columns; more, whose blocks cut tokens in two; one
    # sequence or more than 256; lengths of one tile, of several pieces, of one sequence only
    (128, 32, 8, 64, [(4, 2000 + 37 * i) for i in range(8)], False),
    (128, 8, 2, 16, [(i % 5, 30 + i) for i in range(300)], True),
    (256, 8, 1, 32, [(4, 900), (0, 700), (2, 3), (1, 1)], True),
    (64, 6, 2, 16, [(33, 1200), (1, 40), (7, 5), (33, 33)], False),
    (128, 5, 5, 128, [(16, 5000)], True), (128, 40, 1, 64, [(3, 777), (2, 1)], False),
    (64, 1, 1, 16, [(16, 16), (16, 0), (16, 17), (15, 4000)], False),
    (128, 10, 10, 32, [(128, 900)], True), (256, 4, 4, 16, [(16, 16)] * 60, False),
]


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("D,heads,hk,page,seqs,mask", FEW)
def test_few_tokens(D, heads, hk, page, seqs, mask, fmt):
    test_attention(D, heads, hk, page, seqs, mask, fmt)


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("D,hk,group,n,L", [(128, 2, 4, 4, 70), (64, 1, 3, 5, 3000),
                                            (256, 3, 2, 16, 129), (128, 1, 5, 11, 11)])
def test_few_tokens_not_finite(D, hk, group, n, L, mask, fmt):
    """Values that are not finite among the new tokens and before them, in slots that later tokens see, or nobody."""
    gen = torch.Generator().manual_seed(D + L)
    page = 16
    cache, plain = R.make_cache(gen, 1, L, hk, D, page, fmt)
    plain = rrs.KVCache(plain.k.clone(), plain.v.clone(), plain.table)
    bad = [(L - 1, 2, math.nan), (L - n // 2, 40, math.inf), (L - n + 1, 5, -math.inf),
           (max(L - n - 3, 0), 7, math.nan), (max(L - n - 2, 0), 60, math.inf)]
    m = None
    if mask:
        m = (torch.rand((1, cache.capacity), generator=gen) < 0.7).cuda()
        m[0, L - n + 1], m[0, L - 1] = False, True
    for i, (t, d, what) in enumerate(bad):
        p, at, h = int(cache.table[0, t // page]), t % page, i % hk
        if fmt == "f16":
            cache.v[p, h, at, d] = what
            plain.v[p, h, at, d] = what
        elif fmt == "int4":
            cache.v_scale[p, h, at] = what
            plain.v[p, h, at] = math.nan
        else:
            cache.v.view(torch.uint8)[p, h, at, d] = 127
            plain.v[p, h, at, d] = math.nan
    starts, rows = _starts([n])
    Q = torch.randn((n, group * hk, D), generator=gen).half().cuda()
    out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), mask=m, return_lse=True)
    R.check(out, lse, R.attention(Q, plain, rows, [L], D ** -0.5, m), rows)
    # A key: NaN for the tokens that see it, for the others what was there.
    t = L - 2
    p, at = int(cache.table[0, t // page]), t % page
    if m is not None:
        m[0, t] = True
        out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), mask=m, return_lse=True)
    if fmt == "f16":
        cache.k[p, 0, at, 3] = math.nan
    elif fmt == "int4":
        cache.k_scale[p, 0, at] = math.nan
    else:
        cache.k.view(torch.uint8)[p, 0, at, 3] = 255
    new, new_lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), mask=m, return_lse=True)
    assert bool(new[n - 2:, :group].isnan().all()) and bool(new_lse[n - 2:, :group].isnan().all())
    R.check(new[:n - 2], new_lse[:n - 2],
            R.attention(Q[:n - 2], plain, [(0, n - 2)], [L - 2], D ** -0.5, m), [(0, n - 2)])


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_scale(scale, fmt):
    gen = torch.Generator().manual_seed(3)
    cache, plain = R.make_cache(gen, 2, 200, 2, 128, 32, fmt)
    starts, rows = _starts([40, 9])
    Q = torch.randn((49, 6, 128), generator=gen).half().cuda()
    out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([200, 77]), scale=scale,
                                    return_lse=True)
    R.check(out, lse, R.attention(Q, plain, rows, [200, 77], scale), rows)
    starts, rows = _starts([5, 3])
    out, lse = rrs.prompt_attention(Q[:8], cache, _int(starts), _int([200, 77]), max_tokens=5,
                                    scale=scale, return_lse=True)
    R.check(out, lse, R.attention(Q[:8], plain, rows, [200, 77], scale), rows)


def test_growing_logits():
    """Maxima that move in every tile, and weights far below the largest."""
    gen = torch.Generator().manual_seed(4)
    cache, _ = R.make_cache(gen, 1, 640, 1, 64, 64, "f16")
    ramp = torch.linspace(-8, 8, 640).view(10, 1, 64, 1).half().cuda()
    cache.k[cache.table[0].long()] = ramp.expand(10, 1, 64, 64).contiguous()
    starts, rows = _starts([100])
    Q = torch.randn((100, 2, 64), generator=gen).abs().half().cuda()
    Q[:, 1] *= -1
    out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([640]), return_lse=True)
    R.check(out, lse, R.attention(Q, cache, rows, [640], 0.125), rows)


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("D,hk,pieces", [(128, 2, False), (64, 64, False), (256, 1, True)])
def test_not_finite(D, hk, pieces, fmt):
    """A token whose value is not finite shows in the rows that see it, and in no earlier one."""
    gen = torch.Generator().manual_seed(D)
    n, L, page = 90, 150 if not pieces else 600, 32
    cache, plain = R.make_cache(gen, 1, L, hk, D, page, fmt)
    plain = rrs.KVCache(plain.k.clone(), plain.v.clone(), plain.table)
    # Slots with an infinity, a NaN, one in every channel; the last three are among the new tokens.
    for i, (t, what) in enumerate([(L - 70, math.inf), (L - 40, math.nan), (L - 9, -math.inf)]):
        p, at, h, d = int(cache.table[0, t // page]), t % page, i % hk, 5 + 7 * i
        if fmt == "f16":
            cache.v[p, h, at, d] = what
            plain.v[p, h, at, d] = what
        elif fmt == "fp8":
            cache.v.view(torch.uint8)[p, h, at, d] = 255
            plain.v[p, h, at, d] = math.nan
        else:
            cache.v_scale[p, h, at] = what
            plain.v[p, h, at] = math.nan
    starts, rows = _starts([n])
    Q = torch.randn((n, 2 * hk, D), generator=gen).half().cuda()
    out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), return_lse=True)
    R.check(out, lse, R.attention(Q, plain, rows, [L], D ** -0.5), rows)
    # A key: the rows that see it are NaN as a whole.
    t = L - 30
    p, at = int(cache.table[0, t // page]), t % page
    if fmt == "f16":
        cache.k[p, 0, at, 3] = math.nan
    elif fmt == "fp8":
        cache.k.view(torch.uint8)[p, 0, at, 3] = 127
    else:
        cache.k_scale[p, 0, at] = math.nan
    new, new_lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), return_lse=True)
    assert torch.equal(new[:n - 30].view(torch.int16), out[:n - 30].view(torch.int16))
    assert bool(new[n - 30:, :2].isnan().all()) and bool(new_lse[n - 30:, :2].isnan().all())
    assert torch.equal(new_lse[n - 30:, 2:], lse[n - 30:, 2:])


@pytest.mark.parametrize("bound", [8, 99])
def test_bad_numbers(bound):
    """Rows, counts and lengths out of range are cut; the rest is as without them. Few columns and many."""
    gen = torch.Generator().manual_seed(6)
    cache, plain = R.make_cache(gen, 3, 64, 2, 128, 16, "f16")
    M = 12 + bound
    Q = torch.randn((M, 4, 128), generator=gen).half().cuda()
    # More tokens than slots: the first ones see nothing. A length past the bound. Rows past M.
    out, lse = rrs.prompt_attention(Q, cache, _int([0, 8, 12, M + 79]), _int([5, 1000, -4]),
                                    max_tokens=bound, max_length=64, return_lse=True)
    R.check(out, lse, R.attention(Q, plain, [(0, 8), (8, 4)], [5, 64], 128 ** -0.5),
            [(0, 8), (8, 4)])
    assert not out[12:].any()
    # A table entry that is no page reads as page 0.
    table = cache.table.clone()
    table[0, 1] = -9
    zero = cache.table.clone()
    zero[0, 1] = 0
    starts, n = _int([0, 20, 20, 20]), _int([50, 1, 1])
    got, want = (rrs.prompt_attention(Q, cache._replace(table=t), starts, n,
                                      max_tokens=max(bound, 20))[:20] for t in (table, zero))
    assert torch.equal(got, want)


def test_one_token_is_paged_attention():
    gen = torch.Generator().manual_seed(7)
    for fmt in ("f16", "int4", "fp8"):
        cache, plain = R.make_cache(gen, 5, 300, 2, 128, 32, fmt)
        lengths = [1, 300, 77, 16, 129]
        Q = torch.randn((5, 8, 128), generator=gen).half().cuda()
        starts, rows = _starts([1] * 5)
        ref = R.attention(Q, plain, rows, lengths, 128 ** -0.5)
        out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int(lengths), return_lse=True)
        R.check(out, lse, ref, rows)
        y, l = rrs.paged_attention(Q, cache, _int(lengths), return_lse=True)
        if fmt != "int4":   # paged attention keeps INT4 products exact, prompts round q s to float16
            R.check(y, l, ref, rows)


def test_many_tokens():
    """A tile of rows that ends inside a token's heads, tokens in thousands, a long cache."""
    gen = torch.Generator().manual_seed(8)
    cache, plain = R.make_cache(gen, 1, 2600, 1, 64, 64, "fp8")
    starts, rows = _starts([1100])
    Q = torch.randn((1100, 3, 64), generator=gen).half().cuda()
    out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([2600]), return_lse=True)
    R.check(out, lse, R.attention(Q, plain, rows, [2600], 0.125), rows)


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("bound", [60, 4])
def test_graph(mask, bound):
    """Captured once, replayed over other queries, starts and lengths."""
    gen = torch.Generator().manual_seed(9)
    cache, _ = R.make_cache(gen, 3, 700, 2, 128, 16, "fp8")
    Q = torch.zeros((60, 8, 128), dtype=torch.float16, device="cuda")
    starts, n = _int([0, 0, 0, 0]), _int([1, 1, 1])
    m = torch.ones((3, cache.capacity), dtype=torch.bool, device="cuda") if mask else None

    def call():
        return rrs.prompt_attention(Q, cache, starts, n, max_tokens=bound, max_length=700, mask=m,
                                    return_lse=True)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for s, l in (([0, 60, 60, 60], [700, 3, 9]), ([0, 1, 30, 60], [5, 640, 33]),
                 ([0, 20, 40, 60], [20, 20, 20])):
        s = [x * bound // 60 for x in s]
        Q.copy_(torch.randn(Q.shape, generator=gen))
        starts.copy_(_int(s)), n.copy_(_int(l))
        if mask:
            m.copy_(torch.rand(m.shape, generator=gen) < 0.5)
        graph.replay()
        for x, y in zip(got, call()):
            assert torch.equal(x[:s[3]], y[:s[3]])
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("mask", [False, True])
def test_many_rows(fmt, mask):
    """Bounds of 4096 tokens with 64 heads and 8192 slots take workgroups of eight waves, tight ones of four."""
    gen = torch.Generator().manual_seed(10)
    hk, heads, D, B = 16, 64, 128, 2
    cache, plain = R.make_cache(gen, B, 8192, hk, D, 64, fmt)
    counts, lengths = [70, 3], [640, 77]
    starts, rows = _starts(counts)
    Q = torch.randn((4096, heads, D), generator=gen).half().cuda()
    n, s = _int(lengths), _int(starts)
    m = None
    if mask:
        m = (torch.rand((B, cache.capacity), generator=gen) < 0.7).cuda()
    _fill_dead(cache, n, m, fmt)
    out, lse = rrs.prompt_attention(Q, cache, s, n, mask=m, return_lse=True)
    ref = R.attention(Q, plain, rows, lengths, D ** -0.5, m)
    R.check(out, lse, ref, rows)
    out, lse = rrs.prompt_attention(Q, cache, s, n, max_tokens=70, max_length=640, mask=m,
                                    return_lse=True)
    R.check(out, lse, ref, rows)


@pytest.mark.parametrize("D,hk,L,fmt", [(128, 1, 5003, "fp8"), (256, 2, 3001, "int4"),
                                        (64, 1, 9001, "f16")])
def test_many_pieces(D, hk, L, fmt):
    """A few tokens over one long cache: many pieces, the join by groups of threads; a row without a slot."""
    gen = torch.Generator().manual_seed(D)
    cache, plain = R.make_cache(gen, 1, L, hk, D, 64, fmt)
    starts, rows = _starts([5])
    Q = torch.randn((5, 3 * hk, D), generator=gen).half().cuda()
    m = torch.ones((1, cache.capacity), dtype=torch.bool, device="cuda")
    m[0, :L - 4] = False
    for mask in (None, m):
        out, lse = rrs.prompt_attention(Q, cache, _int(starts), _int([L]), mask=mask,
                                        return_lse=True)
        R.check(out, lse, R.attention(Q, plain, rows, [L], D ** -0.5, mask), rows)
