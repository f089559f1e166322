"""Plain forms of the FP8 cache on the CPU (not collected by pytest)."""
import math

import torch

import paper_2409_20361_amd as rrs

BLOCK = 16
E4M3 = torch.tensor([(-1.0 if c & 128 else 1.0) * (
    math.nan if c & 127 == 127 else
    (c & 7) * 2.0 ** -9 if c & 120 == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
    for c in range(256)], dtype=torch.float64)   # what a code stands for


def encode(x):
    """float64 of magnitude up to 448 (or NaN) -> codes (uint8) of the nearest e4m3 numbers, ties to even."""
    a = x.abs()
    e = torch.clamp(torch.frexp(torch.where(a > 0, a, 2.0 ** -9))[1].double() - 1, min=-6.0)
    q = torch.round(a / torch.exp2(e - 3))               # 0 .. 16 units of the binade
    code = torch.where(a.isnan(), 127.0, (e + 6) * 8 + q).to(torch.uint8)
    return code | (torch.signbit(x).to(torch.uint8) << 7)


def exponent(top):
    """Of the smallest scale from 2^-15 on that brings top to 448 at most."""
    e = -15
    while top > 448 * 2.0 ** e:
        e += 1
    return e


def quantize(x, e):
    """float16 values in float64 -> codes in the scale 2^e."""
    most = 240.0 if e == 8 else 448.0
    return encode(torch.where(x.isfinite(), (x / 2.0 ** e).clamp(-most, most), math.nan))


def append(codes, scales, first, new):
    """One head's block: codes (16, D) uint8, its scale; new (n, D) float64 to slots first... In place;
    returns the scale."""
    so_far = -15 if first == 0 else int(math.log2(float(scales)))
    finite = new[new.isfinite()]
    e = max(so_far, exponent(float(finite.abs().max()) if finite.numel() else 0.0))
    if e > so_far and first:
        codes[:] = encode((E4M3[codes.long()] * 2.0 ** (so_far - e)))
    codes[first:first + len(new)] = quantize(new, e)
    return 2.0 ** e


def make_cache(gen, B, capacity, hk, D, page, extra_pages=3, spread=1.0):
    """A random FP8 cache on the GPU whose pages are in random order, and the float16 cache of the
    same values. spread: of the blocks' sizes, in octaves."""
    per_seq = -(-capacity // page)
    pages = B * per_seq + extra_pages
    table = torch.randperm(pages, generator=gen)[:B * per_seq].view(B, per_seq).int().cuda()
    pools = []
    for _ in range(2):
        x = torch.randn((pages, hk, page // BLOCK, BLOCK * D), generator=gen).half().double()
        x *= torch.exp2(spread * torch.randn(x.shape[:3] + (1,), generator=gen)).half()
        x = x.half().double()
        top = x.abs().amax(-1)
        e = torch.ceil(torch.log2(top / 448)).clamp(min=-15.0)
        codes = encode(x / torch.exp2(e).unsqueeze(-1)).view(pages, hk, page, D)
        scale = torch.exp2(e)
        value = E4M3[codes.long()] * scale.repeat_interleave(BLOCK, -1).unsqueeze(-1)
        assert bool((value.half().double() == value).all())
        pools.append((codes.cuda().view(torch.float8_e4m3fn), scale.half().cuda(),
                      value.half().cuda()))
    (k, ks, k16), (v, vs, v16) = pools
    return rrs.KVCache(k, v, table, ks, vs), rrs.KVCache(k16, v16, table)
