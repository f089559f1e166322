"""Plain 64-bit forms of the key/value cache operators, on the CPU (not collected by pytest)."""
import math

import torch

import paper_2409_20361_amd as rrs


def unpack(codes):
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    return torch.where(q > 7, q - 16, q)


def pack(q):
    q = q.to(torch.int64) & 15
    return (q[..., 0::2] | (q[..., 1::2] << 4)).to(torch.uint8)


def quantize(x):
    """float64 values (of float16) -> codes (int64) and float16 scales, as include/rrs.h states."""
    scale = (x.abs().amax(-1) / 7).half()
    s = scale.double().unsqueeze(-1)
    q = torch.where(s > 0, torch.round(x / torch.where(s > 0, s, 1.0)), 0.0).clamp(-7, 7)
    return q.long(), scale


def make_cache(gen, B, capacity, hk, D, page, fmt, extra_pages=3, fill=None):
    """A random cache on the GPU whose pages are in random order; fill: the value of everything
    (float16 only)."""
    per_seq = -(-capacity // page)
    pages = B * per_seq + extra_pages
    table = torch.randperm(pages, generator=gen)[:B * per_seq].view(B, per_seq).int()
    shape = (pages, hk, page, D)
    x = [torch.randn(shape, generator=gen).half() for _ in range(2)]
    if fmt == "f16":
        if fill is not None:
            x = [torch.full(shape, fill, dtype=torch.float16) for _ in range(2)]
        return rrs.KVCache(x[0].cuda(), x[1].cuda(), table.cuda())
    q = [quantize(v.double()) for v in x]
    return rrs.KVCache(pack(q[0][0]).cuda(), pack(q[1][0]).cuda(), table.cuda(), q[0][1].cuda(),
                       q[1][1].cuda())


def values(cache, b, n):
    """K, V (KV heads, n, D) of sequence b in float64 on the CPU; scales of V (KV heads, n) or None."""
    out, P = [], cache.k.shape[2]
    pages = cache.table[b, :max(1, -(-n // P))].long()
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = pool[pages].cpu().transpose(0, 1)
        x = x.reshape(x.shape[0], -1, x.shape[-1])[:, :n]
        s = None
        if scale is not None:
            s = scale[pages].cpu().transpose(0, 1).reshape(x.shape[0], -1)[:, :n].double()
            x = unpack(x).double() * s.unsqueeze(-1)
        out.append(x.double())
    return out[0], out[1], s


def attention(Q, cache, lengths, scale, mask=None):
    """For each sequence None (no slot takes part) or a dict: o, lse, p, live, and the bounds below.

    With u = 2^-24, the products of q . k summed in any order in float32 are off by at most
    (D + 8) u sum |q k|; with the scale's and the exponent's own roundings a logit is off by
    d = |scale| (D + 8) u max sum |q k| + 4 u max |l|. A weight is then off by 2 d relative
    (it and the sum), plus n u for the sum and 2^-20 for the exponential; in the product with V it may be
    rounded to float16 (2^-11 relative, or half a subnormal step, 2^-25 of the largest
    weight, times the largest |v| of its row; for INT4 the weight carries the row's
    scale). The output is rounded to float16 once more."""
    res = []
    H, D = Q.shape[1:]
    for b, n in enumerate(lengths):
        k, v, s = values(cache, b, n)
        hk = k.shape[0]
        live = torch.ones(n, dtype=torch.bool)
        if mask is not None:
            live = mask[b, :n].cpu().bool()
        if not bool(live.any()):
            res.append(None)
            continue
        k, v = k[:, live], v[:, live]
        q = Q[b].double().cpu().view(hk, H // hk, D)
        logits = q @ k.transpose(1, 2) * scale
        u = 2.0 ** -24
        d = (abs(scale) * (D + 8) * u * (q.abs() @ k.abs().transpose(1, 2)).amax()
             + 4 * u * logits.abs().amax()).item()
        p = torch.softmax(logits, -1)
        o = p @ v
        rel = 2 * d + n * u + 2.0 ** -20
        vmax = v.abs().amax(-1) if s is None else 7 * s[:, live]
        worst = (p * vmax.unsqueeze(1)).amax(-1, keepdim=True)
        tol = ((2.0 ** -11 + rel) * (p @ v.abs()) + (2.0 ** -11 + 2.0 ** -20) * o.abs()
               + 2.0 ** -24 * int(live.sum()) * worst + 2.0 ** -24)
        full = torch.zeros((hk, H // hk, n), dtype=torch.float64)
        full[:, :, live] = p
        lse = torch.logsumexp(logits, -1)
        res.append({"o": o.reshape(H, D), "tol": tol.reshape(H, D), "lse": lse.reshape(H),
                    "lse_tol": rel + 4 * u * lse.abs().amax().item(), "w": full.sum(1),
                    "w_tol": rel * full.sum(1), "live": live})
    return res


def evict(n, budget, weights, pos, keep_from):
    """kept of one (sequence, KV head): a list, by sorting."""
    if n <= budget:
        return list(range(n))

    def key(t):
        w = float(weights[t])
        guard = int(pos[t]) >= keep_from
        return (0 if guard else 1, -math.inf if guard else (math.inf if math.isnan(w) else -w),
                math.isnan(w) and not guard, t)
    keep = set(sorted(range(n), key=key)[:budget])
    late = iter([t for t in range(budget, n) if t in keep])
    return [t if t in keep else next(late) for t in range(budget)]
