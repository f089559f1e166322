"""Plain 64-bit form of prompt attention, on the CPU (not collected by pytest)."""
import math

import torch

import _fp8_util as F
import _kv_util as U
import paper_2409_20361_amd as rrs


def make_cache(gen, B, capacity, hk, D, page, fmt):
    """A random cache on the GPU, and the float16 cache of the values that it stands for."""
    if fmt == "fp8":
        return F.make_cache(gen, B, capacity, hk, D, page)
    cache = U.make_cache(gen, B, capacity, hk, D, page, fmt)
    if fmt == "f16":
        return cache, cache
    k, v = ((U.unpack(x.cpu()).double() * s.cpu().double().unsqueeze(-1)).half().cuda()
            for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    return cache, rrs.KVCache(k, v, cache.table)


def attention(Q, plain, rows, lengths, scale, mask=None):
    """Of every sequence's rows: o (n, H, D), its tolerance, lse (n, H), its tolerance, and which rows see
    anything. Q (M, H, D); rows: the sequences' (first, count).

    With u = 2^-24, the products of q . k summed in any order in float32 are off by at most (D + 8) u
    sum |q k|; with the scale's and the exponent's own roundings a logit is off by
    d = |scale| (D + 8) u max sum |q k| + 4 u max |l|. A weight is then off by 2 d relative (it and
    the sum), plus n u for the sum and 2^-20 for the exponential; in the product with V it may be
    rounded to float16 (2^-11 relative, or half a subnormal step, 2^-25, in units that leave the
    largest weight at 2^12 or more). The output is rounded to float16 once more, by half a step:
    2^-11 relative or 2^-25."""
    res = []
    H, D = Q.shape[1:]
    u = 2.0 ** -24
    for b, ((first, n), L) in enumerate(zip(rows, lengths)):
        if n == 0:
            res.append(None)
            continue
        if L == 0:   # tokens that see nothing
            o, l = torch.zeros((n, H, D)).double(), torch.full((n, H), -math.inf).double()
            res.append({"o": o, "tol": o, "lse": l, "lse_tol": torch.zeros_like(l),
                        "some": torch.zeros(n, dtype=torch.bool)})
            continue
        k, v, _ = U.values(plain, b, L)
        hk = k.shape[0]
        q = Q[first:first + n].double().cpu().view(n, hk, H // hk, D).permute(1, 2, 0, 3)
        live = torch.arange(L) <= torch.arange(L - n, L)[:, None]
        if mask is not None:
            live = live & mask[b, :L].cpu().bool()
        some = live.any(1)
        # Slots that a row does not see count nowhere, whatever they hold.
        seen = live.any(0)
        k = torch.where(seen[:, None], k, 0.0)
        dead = ~live
        logits = (q @ k.transpose(1, 2).unsqueeze(1) * scale)
        size = (q.abs() @ k.abs().transpose(1, 2).unsqueeze(1)).masked_fill(dead, 0.0)
        masked = logits.masked_fill(dead, -math.inf)
        top = logits.masked_fill(dead, 0.0).abs().amax((-1), keepdim=True)
        d = abs(scale) * (D + 8) * u * size.amax(-1, keepdim=True) + 4 * u * top
        p = torch.where(some[:, None], torch.softmax(masked, -1), 0.0)
        lse = torch.logsumexp(masked, -1)
        rel = 2 * d + L * u + 2.0 ** -20
        o = torch.zeros((hk, H // hk, n, D), dtype=torch.float64)
        for t in range(L):   # 0 times what is not finite does not count
            if not bool(seen[t]):
                continue
            if bool(v[:, t].isfinite().all()):
                continue
            x = v[:, t][:, None, None]
            on = live[:, t][None, None, :, None] & ~x.isfinite()
            o += torch.where(on, p[..., t:t + 1] * x, 0.0)
        clean = torch.where(v.isfinite(), v, 0.0).unsqueeze(1)
        o += p @ clean
        size = p @ clean.abs()
        worst = (p * clean.abs().amax(-1).unsqueeze(2)).amax(-1, keepdim=True)
        tol = ((2.0 ** -11 + rel) * size + 2.0 ** -11 * (1 + 2.0 ** -10) * o.abs()
               + L * 2.0 ** -37 * torch.where(p.sum(-1, keepdim=True) > 0, clean.abs().amax(), 0.0)
               + 2.0 ** -24 * worst + 2.0 ** -25)
        lse_tol = rel[..., 0] + 4 * u * lse.abs().masked_fill(~some, 0.0)

        def rows_first(x):
            return x.permute(2, 0, 1, *range(3, x.dim())).reshape(n, H, *x.shape[3:])
        res.append({"o": rows_first(o), "tol": rows_first(tol), "lse": rows_first(lse),
                    "lse_tol": rows_first(lse_tol), "some": some})
    return res


def check(out, lse, ref, rows):
    for (first, n), r in zip(rows, ref):
        if r is None:
            continue
        got = out[first:first + n].double().cpu()
        l = lse[first:first + n].double().cpu()
        some = r["some"]
        assert not got[~some].any() and bool((l[~some] == -math.inf).all())
        want, fine = r["o"], r["o"].isfinite()
        assert bool((got.isfinite() == fine)[some].all())
        bad = torch.where(fine, (got - want).abs() - r["tol"], -1.0)[some]
        assert bool((bad <= 0).all()), (first, n, float(bad.max()))
        err = (l - r["lse"]).abs()[some]
        assert bool((err <= r["lse_tol"][some]).all()), (first, n, float(err.max()))
