"""Workloads of the 8-bit cache, prompts and pages: what is measured, in plain torch and through the package.

  append   rrs.rope_kv_append into an FP8 cache, whose blocks of 16 slots share a scale for each head: a
           block that gets a larger value gets a larger scale, and its older rows new codes; the
           cache is then read back as values (rrs.kv_read)
  attend   rrs.paged_attention: one new token per sequence over its FP8 cache
  prompt   rrs.prompt_attention: causal attention of every sequence's new tokens over its cache
  fork     rrs.kv_fork, rrs.kv_copy_pages: rows of the page table are forked, freed and extended, and
           shared pages that are about to be written are copied
  compact  rrs.kv_compact, rrs.kv_copy_pages: the pages in use move to the front of the pool

Caches: k, v (pages, KV heads, page size, D) float16; or D/2 bytes of packed INT4 codes (low nibble first)
with one float16 scale per token and head; or float8_e4m3fn with one float16 scale, a power of two in
[2^-15, 2^8], per block of 16 slots and head. table (sequences, pages per sequence) int32.
"""
import math
import random

import torch

own = False

BLOCK = 16   # slots that share a scale (FP8)


def _append(M, heads, kv_heads, D, seqs=1, past=0, page=64, rotary=None, name=None):
    c = {"op": "append", "M": M, "heads": heads, "kv_heads": kv_heads, "D": D, "fmt": "fp8",
         "seqs": seqs, "past": past, "page": page, "rotary": D if rotary is None else rotary}
    return c if name is None else {"name": name, **c}


def _attend(B, S, heads, kv_heads, D, page=64, ragged=True, mask=False, weights=False, lse=False,
            name=None):
    c = {"op": "attend", "B": B, "S": S, "heads": heads, "kv_heads": kv_heads, "D": D, "fmt": "fp8",
         "page": page, "ragged": ragged, "mask": mask, "weights": weights, "lse": lse}
    return c if name is None else {"name": name, **c}


def _prompt(B, T, past, heads, kv_heads, D, fmt="fp8", page=64, mask=False, lse=False, name=None):
    c = {"op": "prompt", "B": B, "T": T, "past": past, "heads": heads, "kv_heads": kv_heads, "D": D,
         "fmt": fmt, "page": page, "mask": mask, "lse": lse}
    return c if name is None else {"name": name, **c}


def _fork(groups, width, S, grow, kv_heads, D, fmt="f16", page=64, name=None):
    c = {"op": "fork", "groups": groups, "width": width, "S": S, "grow": grow, "kv_heads": kv_heads,
         "D": D, "fmt": fmt, "page": page}
    return c if name is None else {"name": name, **c}


def _compact(B, S, fill, kv_heads, D, fmt="f16", page=64, name=None):
    c = {"op": "compact", "B": B, "S": S, "fill": fill, "kv_heads": kv_heads, "D": D, "fmt": fmt,
         "page": page}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One token of one sequence in the middle of a block: latency.
        _append(1, 32, 8, 128, past=517, name="append_1"),
        # Prompts of odd lengths, behind what their sequences hold already.
        _append(6113, 32, 32, 128, seqs=7, past=41, page=32, name="append_6113"),
        # One sequence a short way into its answer: latency.
        _attend(1, 213, 32, 32, 128, name="attend_1"),
        # A decode batch of sequences of all ages.
        _attend(64, 8192, 32, 8, 128, page=32, name="attend_64"),
        # One sequence at the end of a very long context, some of its tokens masked out.
        _attend(1, 131071, 64, 8, 128, mask=True, lse=True, name="attend_long"),
        # A few proposed tokens per sequence, to be verified in one pass.
        _prompt(9, 7, 1501, 20, 5, 64, "f16", page=16, name="prompt_9_f16"),
        # The next part of a long prompt, over what is cached of it in 4 bits.
        _prompt(1, 1024, 12288, 32, 8, 128, "int4", lse=True, name="prompt_1024_int4"),
        # Whole prompts of a batch.
        _prompt(4, 8192, 0, 32, 8, 128, name="prompt_8192"),
        # Beams of one prompt, one step: latency.
        _fork(1, 8, 700, 1, 8, 128, page=16, name="fork_8"),
        # Samples of many prompts, one step.
        _fork(64, 4, 4096, 1, 8, 128, page=64, name="fork_256"),
        # A small pool with a few holes: latency.
        _compact(5, 300, 0.8, 8, 128, page=16, name="compact_5"),
        # A large pool that is to be cut to what is in use.
        _compact(128, 4096, 0.55, 8, 128, page=64, name="compact_128"),
    ]


_HEADS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (20, 5, 64), (32, 32, 64), (40, 1, 256),
          (16, 8, 256), (9, 3, 128), (40, 1, 64)]
_MAX_APPEND = 6113 * 12288
_MAX_CACHE = 64 * 8192 * 8 * 128
_MAX_FLOPS = 4 * 4 * 8192 * 4096 * 128 * 32 // 2
_MAX_POOL = 64 * 4 * 4096 * 8 * 128 // 4


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "prompt", "prompt", "fork", "compact"])
        H, Hk, D = rng.choice(_HEADS)
        fmt = rng.choice(["f16", "int4", "fp8"])
        page = rng.choice([16, 32, 64, 128, 256])
        if op == "append":
            M = _log_int(rng, 1, 6113)
            seqs, past = min(M, _log_int(rng, 1, 64)), rng.choice([0, _log_int(rng, 1, 2048)])
            rotary = rng.choice([D, D, D // 2, D // 4])
            if M * (H + 2 * Hk) * D <= _MAX_APPEND and seqs * (past + M) * Hk * D <= _MAX_CACHE // 8:
                return _append(M, H, Hk, D, seqs, past, page, rotary)
        elif op == "attend":
            B, S = _log_int(rng, 1, 256), _log_int(rng, 1, 131072)
            if B * S * Hk * D <= _MAX_CACHE:
                return _attend(B, S, H, Hk, D, page, rng.random() < 0.7, rng.random() < 0.2,
                               rng.random() < 0.3, rng.random() < 0.5)
        elif op == "prompt":
            B, T = _log_int(rng, 1, 32), _log_int(rng, 1, 8192)
            past = rng.choice([0, _log_int(rng, 1, 16384)])
            if (4 * B * T * (past + T) * D * H <= _MAX_FLOPS
                    and B * (past + T) * Hk * D <= _MAX_CACHE // 2):
                return _prompt(B, T, past, H, Hk, D, fmt, page, rng.random() < 0.2,
                               rng.random() < 0.3)
        elif op == "fork":
            G, W, S = _log_int(rng, 1, 64), _log_int(rng, 1, 32), _log_int(rng, 1, 16384)
            if G * W * S * Hk * D <= _MAX_POOL:
                return _fork(G, W, S, rng.choice([1, 1, 1, 7, page, 5 * page + 3]), Hk, D, fmt, page)
        else:
            B, S = _log_int(rng, 1, 256), _log_int(rng, 1, 32768)
            fill = rng.uniform(0.3, 0.98)
            if B * S * Hk * D <= _MAX_POOL * fill:
                return _compact(B, S, fill, Hk, D, fmt, page)


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------

def _counts(M, seqs):
    """New tokens of each sequence: a ragged partition of M, at least one each."""
    cuts = sorted(random.Random(11 * M + seqs).sample(range(1, M), seqs - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [M])]


def _lengths(B, S, ragged=True):
    """Lengths of a batch: the longest is S, the others spread from one token on."""
    if not ragged:
        return [S] * B
    r = random.Random(13 * B + S)
    return [S] + [r.randint(1, S) for _ in range(B - 1)]


def _prompt_lengths(case):
    """New tokens and cached ones of each sequence."""
    r = random.Random(17 * case["B"] + 19 * case["T"] + case["past"])
    new = [case["T"]] + [r.randint(1, case["T"]) for _ in range(case["B"] - 1)]
    return new, [case["past"]] + [r.randint(0, case["past"]) for _ in range(case["B"] - 1)]


def _beams(case):
    """Of every group its length, how many tokens its rows have in common, and which row of the group
    each row continues (-1 for all: the group has ended)."""
    r = random.Random(23 * case["groups"] + 29 * case["width"] + case["S"])
    W, groups = case["width"], []
    for n in _lengths(case["groups"], case["S"]):
        ended = len(groups) > 0 and r.random() < 0.06
        groups.append((n, r.randint(n // 2, n),
                       [-1 if ended else r.randrange(W) for _ in range(W)]))
    return groups


def _copies(case):
    """Pages that have to be copied: of the rows that continue the same row, all but one."""
    return sum(len(parents) - len(set(parents)) for n, _, parents in _beams(case)
               if n % case["page"] != 0 and parents[0] >= 0)


def _randn(gen, *shape, dtype=torch.float16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pools(case, gen, pages):
    """k, v, k_scale, v_scale of a cache."""
    Hk, D, P = case["kv_heads"], case["D"], case["page"]
    outlier = torch.exp(0.5 * _randn(gen, Hk, 1, D))   # a few key channels are much larger
    k, v = _randn(gen, pages, Hk, P, D).mul_(outlier), _randn(gen, pages, Hk, P, D)
    if case["fmt"] == "f16":
        return k, v, None, None
    out = []
    for x in (k, v):
        if case["fmt"] == "int4":
            scale = (x.abs().amax(-1).float() / 7.0).half()
            q = (x.float() / scale.float().unsqueeze(-1)).round_().clamp_(-7, 7).to(torch.int8)
            out.append((((q[..., 0::2] & 15) | (q[..., 1::2] << 4)).view(torch.uint8), scale))
        else:
            x = x.view(pages, Hk, P // BLOCK, BLOCK * D)
            scale = _block_scale(x.abs().amax(-1).float())
            codes = (x / scale.unsqueeze(-1).half()).to(torch.float8_e4m3fn)
            out.append((codes.view(pages, Hk, P, D), scale.half()))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _batch_cache(case, gen, seqs, capacity):
    """The five tensors of a cache whose pages lie in any order."""
    per_seq = -(-capacity // case["page"])
    table = torch.randperm(seqs * per_seq, generator=gen, device="cuda").to(torch.int32)
    k, v, k_scale, v_scale = _pools(case, gen, seqs * per_seq)
    return k, v, table.view(seqs, per_seq), k_scale, v_scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000033 * seed + 31)
    return {"append": _prepare_append, "attend": _prepare_attend, "prompt": _prepare_prompt,
            "fork": _prepare_fork, "compact": _prepare_compact}[case["op"]](case, gen, seed)


def _prepare_append(case, gen, seed):
    M, H, Hk, D = case["M"], case["heads"], case["kv_heads"], case["D"]
    counts, past = _counts(M, case["seqs"]), case["past"]
    top = past + max(counts)
    s = {"case": case, "cache": _batch_cache(case, gen, case["seqs"], top), "max_length": top}
    s["qkv"] = _randn(gen, M, (H + 2 * Hk) * D)
    s["qkv"][:, ::97] *= 8.0
    s["qkv"] *= torch.exp(_randn(gen, M, 1))   # tokens of different size: scales grow
    rank = torch.cat([torch.arange(n) for n in counts]).cuda()
    s["seq"] = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)
                                       ).to(torch.int32).cuda()
    s["slot"] = (rank + past).to(torch.int32)
    s["positions"] = s["slot"].view(-1, 1).contiguous()
    F = case["rotary"] // 2
    inv = 10000.0 ** (-torch.arange(F, device="cuda", dtype=torch.float64) / F)
    angle = torch.arange(top, device="cuda", dtype=torch.float64)[:, None] * inv
    s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    s["lengths"] = _int32([past + n for n in counts])
    return s


def _prepare_attend(case, gen, seed):
    B, S = case["B"], case["S"]
    lengths = _lengths(B, S, case["ragged"])
    random.Random(seed).shuffle(lengths)
    s = {"case": case, "cache": _batch_cache(case, gen, B, S), "lengths": _int32(lengths),
         "q": _randn(gen, B, case["heads"], case["D"]), "mask": None, "weights": None}
    capacity = s["cache"][2].shape[1] * case["page"]
    if case["mask"]:
        s["mask"] = torch.rand((B, capacity), generator=gen, device="cuda") < 0.8
        if B > 1:
            s["mask"][0] = False
    if case["weights"]:
        s["weights"] = _randn(gen, B, case["kv_heads"], capacity, dtype=torch.float32).abs_()
    return s


def _prepare_prompt(case, gen, seed):
    B = case["B"]
    pairs = list(zip(*_prompt_lengths(case)))
    random.Random(seed).shuffle(pairs)
    new, total = [n for n, _ in pairs], [n + p for n, p in pairs]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s = {"case": case, "new": new, "total": total, "row_start": _int32(starts),
         "lengths": _int32(total), "cache": _batch_cache(case, gen, B, max(total)),
         "q": _randn(gen, starts[-1], case["heads"], case["D"]), "mask": None}
    if case["mask"]:
        capacity = s["cache"][2].shape[1] * case["page"]
        s["mask"] = torch.rand((B, capacity), generator=gen, device="cuda") < 0.8
        s["mask"][:, 0] = False   # the first tokens see nothing
    return s


def _prepare_fork(case, gen, seed):
    P, W = case["page"], case["width"]
    groups = _beams(case)
    order = list(range(len(groups)))
    random.Random(seed).shuffle(order)
    capacity = case["S"] + case["grow"]
    per_row = -(-capacity // P)
    # Every group: pages in common, then each row's own; room for all rows to grow.
    pages = sum(c // P + W * (-(-n // P) - c // P) for n, c, _ in groups)
    pages += W * len(groups) * (-(-case["grow"] // P) + 1)
    free = torch.randperm(pages, generator=gen, device="cuda").tolist()
    rows, lengths, parent = [], [], []
    for g in order:
        n, common, parents = groups[g]
        shared = [free.pop() for _ in range(common // P)]
        base = len(rows)
        for w in range(W):
            row = shared + [free.pop() for _ in range(-(-n // P) - len(shared))]
            rows.append(row + [-1] * (per_row - len(row)))
            lengths.append(n)
            parent.append(base + parents[w] if parents[w] >= 0 else -1)
    k, v, k_scale, v_scale = _pools(case, gen, pages)
    room = [lengths[p] + case["grow"] if p >= 0 else 0 for p in parent]
    return {"case": case, "cache": (k, v, _int32(rows), k_scale, v_scale), "pages": pages,
            "lengths": _int32(lengths), "parent": _int32(parent), "room": _int32(room)}


def _compact_pages(case):
    used = sum(-(-n // case["page"]) for n in _lengths(case["B"], case["S"]))
    return used, max(used, int(used / case["fill"]))


def _prepare_compact(case, gen, seed):
    P = case["page"]
    lengths = _lengths(case["B"], case["S"])
    random.Random(seed).shuffle(lengths)
    used, pages = _compact_pages(case)
    ids = torch.randperm(pages, generator=gen, device="cuda").tolist()
    per_row = -(-case["S"] // P)
    rows = []
    for n in lengths:
        row = [ids.pop() for _ in range(-(-n // P))]
        rows.append(row + [-1] * (per_row - len(row)))
    k, v, k_scale, v_scale = _pools(case, gen, pages)
    return {"case": case, "cache": (k, v, _int32(rows), k_scale, v_scale), "pages": pages,
            "lengths": _int32(lengths)}


# ---------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------

def _block_scale(top):
    """The smallest power of two from 2^-15 on that brings the largest |x| of a block to 448."""
    m, e = torch.frexp(top)                       # 448 = 0.875 * 2^9
    e = torch.where(top > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, -15))
    return torch.ldexp(torch.ones_like(top), e.clamp(min=-15))


def _codes8(x, scale):
    """x / scale as e4m3, in 32 bits; scale 2^8 up to 240, so that code * scale is a float16."""
    q = x / scale
    q = torch.where(scale == 256.0, q.clamp(-240.0, 240.0), q)
    return q.to(torch.float8_e4m3fn).float()


def _unpack(codes, scale):
    """Packed INT4 codes (..., D/2) and their scales (...) as values (..., D)."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    return ((q.to(torch.int16) ^ 8) - 8).float() * scale.float().unsqueeze(-1)


def _values(pool, scale, table, S, fmt):
    """A cache's values (sequences, KV heads, S, D) in 32 bits."""
    table = table.clamp(min=0).long()

    def rows(t, n):
        t = (t.view(torch.uint8)[table].view(t.dtype) if t.dtype == torch.float8_e4m3fn
             else t[table]).transpose(1, 2)
        return t.reshape(t.shape[0], t.shape[1], -1, *t.shape[4:])[:, :, :n]
    if fmt == "f16":
        return rows(pool, S).float()
    if fmt == "int4":
        return _unpack(rows(pool, S), rows(scale, S))
    s = rows(scale, -(-S // BLOCK)).float().repeat_interleave(BLOCK, 2)[:, :, :S]
    return rows(pool, S).float() * s.unsqueeze(-1)


def _read_back(cache, table, lengths, S, fmt):
    live = (torch.arange(S, device="cuda") < lengths[:, None])[:, None, :, None]
    return {"k": torch.where(live, _values(cache[0], cache[3], table, S, fmt), 0.0).half(),
            "v": torch.where(live, _values(cache[1], cache[4], table, S, fmt), 0.0).half()}


def _rotate(x, c, s, R):
    """x (M, heads, D) with its first R dimensions rotated."""
    y = x.clone()
    a, b = x[..., :R // 2], x[..., R // 2:R]
    y[..., :R // 2] = a * c - b * s
    y[..., R // 2:R] = b * c + a * s
    return y


def _plain_append(s):
    case, (k, v, table, k_scale, v_scale) = s["case"], s["cache"]
    M, H, Hk, D, P = case["M"], case["heads"], case["kv_heads"], case["D"], case["page"]
    R = case["rotary"]
    x = s["qkv"].float().view(M, H + 2 * Hk, D)
    p = s["positions"][:, 0].long()
    c, sn = s["rope"][p, None, :R // 2], s["rope"][p, None, R // 2:]
    qk = _rotate(x[:, :H + Hk], c, sn, R).half()
    # The blocks that get new tokens, and more of the same sequences: (seqs, n blocks).
    seq, slot = s["seq"].long(), s["slot"].long()
    b0 = case["past"] // BLOCK
    n = -(-s["max_length"] // BLOCK) - b0
    blocks = torch.arange(b0, b0 + n, device="cuda")
    page = table[:, blocks // (P // BLOCK)].long()
    at = (blocks % (P // BLOCK)).expand_as(page)
    of = seq * n + slot // BLOCK - b0
    written = torch.zeros((case["seqs"] * n, BLOCK), dtype=torch.bool, device="cuda")
    written[of, slot % BLOCK] = True
    fresh = written[:, 0].view(-1, n, 1)
    written = written.view(-1, n, 1, BLOCK, 1)
    for pool, scale, new in ((k, k_scale, qk[:, H:].float()), (v, v_scale, x[:, H + Hk:])):
        top = torch.zeros((case["seqs"] * n, Hk), device="cuda")
        top.scatter_reduce_(0, of[:, None].expand(M, Hk), new.abs().amax(-1), "amax")
        old = torch.where(fresh, 2.0 ** -15, scale[page, :, at].float())
        s_new = torch.maximum(old, _block_scale(top).view(-1, n, Hk))
        touched = written.any(3).view(-1, n, 1)
        s_new = torch.where(touched, s_new, scale[page, :, at].float())
        # (seqs, n, Hk, slots of the block, D)
        slots = at.unsqueeze(-1) * BLOCK + torch.arange(BLOCK, device="cuda")
        codes = pool.view(torch.uint8)[page.unsqueeze(-1), :, slots].view(pool.dtype)
        rows = codes.float().transpose(2, 3)
        grown = _codes8(rows * old[..., None, None], s_new[..., None, None])
        moved = (s_new > old) & touched & ~fresh
        rows = torch.where(moved[..., None, None] & ~written, grown, rows)
        rows = rows.transpose(2, 3).reshape(-1, BLOCK, Hk, D)
        rows[of, slot % BLOCK] = _codes8(new, s_new.view(-1, Hk)[of].unsqueeze(-1))
        rows = rows.view(*codes.shape).to(pool.dtype)
        pool.view(torch.uint8)[page.unsqueeze(-1), :, slots] = rows.view(torch.uint8)
        scale[page, :, at] = s_new.half()
    return {"q": qk[:, :H].contiguous(),
            **_read_back(s["cache"], table, s["lengths"], s["max_length"], "fp8")}


def _softmax(logits, live):
    """Probabilities over the last axis, zeros where nothing is live; and the log of the sum."""
    logits = torch.where(live, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.where(live, torch.exp(logits - torch.where(top > -math.inf, top, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, 1.0), (top + torch.log(total)).squeeze(-1)


def _plain_attend(s):
    case, (k, v, table, k_scale, v_scale) = s["case"], s["cache"]
    B, S, H, Hk, D = case["B"], case["S"], case["heads"], case["kv_heads"], case["D"]
    q = s["q"].float().view(B, Hk, H // Hk, D)
    logits = torch.matmul(q, _values(k, k_scale, table, S, "fp8").transpose(-1, -2)) / math.sqrt(D)
    live = (torch.arange(S, device="cuda") < s["lengths"][:, None])
    if s["mask"] is not None:
        live = live & s["mask"][:, :S]
    p, lse = _softmax(logits, live[:, None, None, :])
    out = {"out": torch.matmul(p, _values(v, v_scale, table, S, "fp8")).view(B, H, D).half()}
    if s["weights"] is not None:
        s["weights"][..., :S] += p.sum(2)
        out["weights"] = s["weights"]
    if case["lse"]:
        out["lse"] = lse.view(B, H)
    return out


def _plain_prompt(s):
    case, (k, v, table, k_scale, v_scale) = s["case"], s["cache"]
    H, Hk, D, fmt = case["heads"], case["kv_heads"], case["D"], case["fmt"]
    G, row, outs, lses = H // Hk, 0, [], []
    for b, (n, S) in enumerate(zip(s["new"], s["total"])):
        q = s["q"][row:row + n].float().view(n, Hk, G, D).permute(1, 2, 0, 3)
        row += n
        keys = _values(k, k_scale, table[b:b + 1], S, fmt)[0].half().float()
        vals = _values(v, v_scale, table[b:b + 1], S, fmt)[0].half().float()
        seen = torch.arange(S, device="cuda") <= torch.arange(S - n, S, device="cuda")[:, None]
        if s["mask"] is not None:
            seen = seen & s["mask"][b, :S]
        step = max(1, (1 << 28) // (G * n * S))   # KV heads at a time
        o, l = [], []
        for h in range(0, Hk, step):
            logits = torch.matmul(q[h:h + step], keys[h:h + step, None].transpose(-1, -2))
            p, lse = _softmax(logits / math.sqrt(D), seen)
            o.append(torch.matmul(p, vals[h:h + step, None]).half())
            l.append(lse)
        outs.append(torch.cat(o).permute(2, 0, 1, 3).reshape(n, H, D))
        lses.append(torch.cat(l).permute(2, 0, 1).reshape(n, H))
    out = {"out": torch.cat(outs)}
    return {**out, "lse": torch.cat(lses)} if case["lse"] else out


def _plain_copy(cache, src, dst, count):
    """Pages src to dst, of the pairs below count."""
    on = torch.arange(src.shape[0], device="cuda") < count
    src, dst = src[on].long(), dst[on].long()
    for t in (cache[0], cache[1], cache[3], cache[4]):
        if t is not None:
            t = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
            t[dst] = t[src]


def _ordered(on, rank, values, size):
    """values where on, at their rank; -1 behind them."""
    out = torch.full((size + 1,), -1, dtype=torch.long, device="cuda")
    return out.scatter_(0, torch.where(on, rank, size), values)[:size]


def _plain_fork(s):
    case, table, pages = s["case"], s["cache"][2].long(), s["pages"]
    S, C, P = *table.shape, case["page"]
    parent, n = s["parent"].long(), s["lengths"].long()
    some = (parent >= 0) & (parent < S)
    p = torch.where(some, parent, 0)
    want = torch.where(some, s["room"].long().clamp(0, C * P), 0)
    kept = torch.minimum(n[p], want)
    old, at = table[p], torch.arange(C, device="cuda")
    have = (kept + P - 1) // P
    live = at < have[:, None]
    refs = torch.zeros(pages + 1, dtype=torch.long, device="cuda")
    refs.scatter_add_(0, torch.where(live, old, pages).flatten(), torch.ones_like(old).flatten())
    refs = refs[:pages]
    # Rows that write into a partly filled page of others too get a page of their own, but for the
    # first of them where nobody else keeps that page.
    rows = torch.arange(S, device="cuda")
    writes = (want > kept) & (kept % P != 0)
    last = old.gather(1, (kept // P).clamp(max=C - 1)[:, None])[:, 0]
    last = torch.where(writes, last, pages)
    writers = torch.zeros(pages + 1, dtype=torch.long, device="cuda")
    writers.scatter_add_(0, last, torch.ones_like(last))
    first = torch.full((pages + 1,), S, dtype=torch.long, device="cuda")
    first.scatter_reduce_(0, last, rows, "amin")
    shared = writes & (torch.cat([refs, refs[:1]])[last] > 1)
    stays = (torch.cat([refs, refs[:1]])[last] == writers[last]) & (first[last] == rows)
    grown = (want + P - 1) // P - have
    left = pages - (refs > 0).sum()
    copy = shared & ~stays
    copy = torch.where((grown + copy).sum() > left, shared, copy)
    need = grown + copy
    upto = need.cumsum(0)
    served = (need == 0) | (upto <= left)
    copy = copy & served
    free = torch.argsort((refs > 0).to(torch.uint8), stable=True)
    begin = upto - need
    fresh = begin[:, None] + copy[:, None] + at - have[:, None]
    fresh = free[fresh.clamp(0, pages - 1)]
    more = ~live & (at < ((want + P - 1) // P)[:, None]) & served[:, None]
    new = torch.where(live, old, torch.where(more, fresh, -1))
    instead = free[begin.clamp(max=pages - 1)]
    new = torch.where(copy[:, None] & (at == (kept // P)[:, None]), instead[:, None], new)
    rank = copy.cumsum(0) - 1
    src, dst = _ordered(copy, rank, last, S), _ordered(copy, rank, instead, S)
    taken = torch.where(served, need, 0).sum()
    i32 = torch.int32
    return {"table": new.to(i32), "lengths": kept.to(i32),
            "room": torch.where(served, want, kept).to(i32), "src": src.to(i32),
            "dst": dst.to(i32), "count": torch.stack([copy.sum(), left - taken]).to(i32)}


def _plain_compact(s):
    case, table, pages = s["case"], s["cache"][2].long(), s["pages"]
    C, P = table.shape[1], case["page"]
    live = torch.arange(C, device="cuda") < ((s["lengths"].long() + P - 1) // P)[:, None]
    used = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    used[torch.where(live, table, pages)] = True
    used = used[:pages]
    U = used.sum()
    ids = torch.arange(pages, device="cuda")
    moves, holes = used & (ids >= U), ~used & (ids < U)
    size = max(1, pages // 2)
    src = _ordered(moves, moves.cumsum(0) - 1, ids, size)
    dst = _ordered(holes, holes.cumsum(0) - 1, ids, size)
    to = torch.where(moves, dst[(moves.cumsum(0) - 1).clamp(0, size - 1)], ids)
    new = torch.where(live, to[torch.where(live, table, 0)], -1)
    i32 = torch.int32
    return {"table": new.to(i32), "src": src.to(i32), "dst": dst.to(i32),
            "count": torch.stack([moves.sum(), U]).to(i32)}


def _pages_out(s, plan, cache):
    """The plan and the cache after the copies: the pools, or what rows of codes stand for."""
    if s["case"]["fmt"] == "f16":
        return {**plan, "k": cache[0], "v": cache[1]}
    lengths = plan.get("lengths", s["lengths"])
    top = s["case"]["S"]
    if own:
        import paper_2409_20361_amd as rrs
        k, v = rrs.kv_read(rrs.KVCache(cache[0], cache[1], plan["table"], cache[3], cache[4]),
                           lengths, top)
        return {**plan, "k": k, "v": v}
    return {**plan, **_read_back(cache, plan["table"], lengths, top, s["case"]["fmt"])}


def _plain_pages(s):
    plan = (_plain_fork if s["case"]["op"] == "fork" else _plain_compact)(s)
    _plain_copy(s["cache"], plan["src"], plan["dst"], plan["count"][0])
    return _pages_out(s, plan, s["cache"])


# ---------------------------------------------------------------------------------------------
# The package's operators
# ---------------------------------------------------------------------------------------------

def _own(s):
    import paper_2409_20361_amd as rrs
    case, cache = s["case"], rrs.KVCache(*s["cache"])
    if case["op"] == "append":
        q = rrs.rope_kv_append(s["qkv"], s["positions"], s["rope"], cache, s["seq"], s["slot"],
                               case["heads"])
        k, v = rrs.kv_read(cache, s["lengths"], s["max_length"])
        return {"q": q, "k": k, "v": v}
    if case["op"] == "attend":
        r = rrs.paged_attention(s["q"], cache, s["lengths"], max_length=case["S"], mask=s["mask"],
                                weights=s["weights"], return_lse=case["lse"])
        out = dict(zip(("out", "lse"), r)) if case["lse"] else {"out": r}
        return out if s["weights"] is None else {**out, "weights": s["weights"]}
    if case["op"] == "prompt":
        r = rrs.prompt_attention(s["q"], cache, s["row_start"], s["lengths"],
                                 max_tokens=max(s["new"]), max_length=max(s["total"]),
                                 mask=s["mask"], return_lse=case["lse"])
        return dict(zip(("out", "lse"), r)) if case["lse"] else {"out": r}
    if case["op"] == "fork":
        plan = rrs.kv_fork(cache.table, s["lengths"], s["parent"], s["room"], s["pages"],
                           case["page"])
        plan = dict(zip(("table", "lengths", "room", "src", "dst", "count"), plan))
    else:
        plan = rrs.kv_compact(cache.table, s["lengths"], s["pages"], case["page"])
        plan = dict(zip(("table", "src", "dst", "count"), plan))
    rrs.kv_copy_pages(cache, plan["src"], plan["dst"], plan["count"])
    return _pages_out(s, plan, cache)


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "prompt": _plain_prompt,
            "fork": _plain_pages, "compact": _plain_pages}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------

def _row_bytes(case):
    """One head's token in k or v, its share of the scale included."""
    D = case["D"]
    return {"f16": 2 * D, "int4": D // 2 + 2, "fp8": D + 2 / BLOCK}[case["fmt"]]


def work(case):
    D, Hk, P, row = case["D"], case["kv_heads"], case["page"], _row_bytes(case)
    if case["op"] == "append":
        M, H, R = case["M"], case["heads"], case["rotary"]
        counts = _counts(M, case["seqs"])
        n = M + case["seqs"] * case["past"]
        nbytes = M * (2 * D * (2 * H + 2 * Hk) + 2 * Hk * row + 4 * (3 + R))
        nbytes += 2 * Hk * (n * row + len(counts) * (case["past"] + max(counts)) * 2 * D)
        return {"bytes": int(nbytes), "flops": 3 * M * (H + Hk) * R}
    if case["op"] == "attend":
        lengths = _lengths(case["B"], case["S"], case["ragged"])
        B, n, H = case["B"], sum(lengths), case["heads"]
        nbytes = 2 * n * Hk * row + 4 * B * H * D + 4 * B + (n if case["mask"] else 0)
        nbytes += (8 * n * Hk if case["weights"] else 0) + (4 * B * H if case["lse"] else 0)
        return {"bytes": int(nbytes), "flops": 4 * n * H * D}
    if case["op"] == "prompt":
        new, past = _prompt_lengths(case)
        H, M, n = case["heads"], sum(new), sum(new) + sum(past)
        nbytes = 2 * n * Hk * row + 4 * M * H * D + (n if case["mask"] else 0)
        pairs = sum(m * p + m * (m + 1) // 2 for m, p in zip(new, past))
        return {"bytes": int(nbytes + (4 * M * H if case["lse"] else 0)),
                "flops": 4 * D * H * pairs}
    if case["op"] == "fork":
        S, moves = case["groups"] * case["width"], _copies(case)
        entries = S * -(-(case["S"] + case["grow"]) // P)
        nbytes = 8 * entries + 4 * S * 7
        slots, rows = sum(n * case["width"] for n, _, _ in _beams(case)), S * case["S"]
    else:
        used, pages = _compact_pages(case)
        moves = used * (pages - used) / pages
        entries = case["B"] * -(-case["S"] // P)
        nbytes = 8 * entries + 4 * case["B"] + 8 * max(1, pages // 2)
        slots, rows = sum(_lengths(case["B"], case["S"])), case["B"] * case["S"]
    nbytes += moves * 4 * Hk * P * row
    if case["fmt"] != "f16":   # read back
        nbytes += 2 * Hk * (slots * row + rows * 2 * D)
    return {"bytes": int(nbytes), "flops": entries}


# ---------------------------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------------------------

def _rows64(cache, b, S, fmt):
    """Keys and values (KV heads, S, D) of one sequence, as the float16 that rows of codes give."""
    k, v, table, k_scale, v_scale = cache
    out = []
    need = table[b].tolist()[:-(-S // k.shape[2])]
    for pool, scale in ((k, k_scale), (v, v_scale)):
        x = torch.cat([pool[p] for p in need], 1)[:, :S]
        if fmt == "f16":
            out.append(x.double())
            continue
        f = torch.cat([scale[p] for p in need], 1).double()
        if fmt == "int4":
            lo, hi = (x & 15).long(), (x >> 4).long()
            x = torch.stack([lo, hi], -1).flatten(-2)
            x = torch.where(x > 7, x - 16, x)
            out.append(x.double() * f[:, :S, None])
        else:
            i = torch.arange(S, device="cuda") // BLOCK
            out.append(x.double() * f[:, i, None])
    return out


def _exact_attend(case, s):
    B, H, Hk, D = case["B"], case["heads"], case["kv_heads"], case["D"]
    outs, lses = [], []
    weights = s["weights"].double() if s["weights"] is not None else None
    for b, n in enumerate(s["lengths"].tolist()):
        k, v = _rows64(s["cache"], b, n, "fp8")
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        if s["mask"] is not None:
            keep = s["mask"][b, :n]
        if not bool(keep.any()):
            outs.append(torch.zeros((H, D), dtype=torch.float64, device="cuda"))
            lses.append(torch.full((H,), -math.inf, dtype=torch.float64, device="cuda"))
            continue
        logits = s["q"][b].double().view(Hk, H // Hk, D) @ k.transpose(1, 2).contiguous()
        logits = (logits * D ** -0.5).masked_fill(~keep, -math.inf)
        p = torch.softmax(logits, -1)
        outs.append((p @ v).reshape(H, D))
        lses.append(torch.logsumexp(logits, -1).reshape(H))
        if weights is not None:
            weights[b, :, :n] += p.sum(1)
    out = {"out": torch.stack(outs)}
    if weights is not None:
        out["weights"] = weights
    if case["lse"]:
        out["lse"] = torch.stack(lses)
    return out


def _exact_prompt(case, s):
    H, Hk, D = case["heads"], case["kv_heads"], case["D"]
    G, row = H // Hk, 0
    M = s["q"].shape[0]
    out = torch.zeros((M, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((M, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, S) in enumerate(zip(s["new"], s["total"])):
        k, v = _rows64(s["cache"], b, S, case["fmt"])
        if case["fmt"] == "int4":   # the values are float16: prompts see what kv_read gives
            k, v = k.half().double(), v.half().double()
        limit = torch.arange(S - n + 1, S + 1, device="cuda")
        rows = max(1, (1 << 27) // S)
        for i in range(0, n, rows):
            m = min(rows, n - i)
            dead = torch.arange(S, device="cuda")[None, :] >= limit[i:i + m, None]
            if s["mask"] is not None:
                dead = dead | ~s["mask"][b, None, :S]
            none = dead.all(1)
            for h in range(H):
                q = s["q"][row + i:row + i + m, h].double()
                logits = (q @ k[h // G].T.contiguous()).mul_(D ** -0.5).masked_fill_(dead, -math.inf)
                at = slice(row + i, row + i + m)
                lse[at, h] = torch.logsumexp(logits, -1)
                p = torch.softmax(logits, -1)
                out[at, h] = torch.where(none[:, None], 0.0, p @ v[h // G])
        row += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _e4m3(x):
    """x to the nearest e4m3 value, ties to even."""
    e = torch.frexp(x)[1].double() - 1
    step = torch.exp2(torch.clamp(e, min=-6.0) - 3)
    return torch.round(x / step) * step


def _exact_append(case, s):
    M, H, Hk, D = case["M"], case["heads"], case["kv_heads"], case["D"]
    R, F = case["rotary"], case["rotary"] // 2
    x = s["qkv"].double().view(M, H + 2 * Hk, D)
    p = s["positions"][:, 0].long()
    cos, sin = s["rope"][p, :F].double()[:, None], s["rope"][p, F:].double()[:, None]
    y = x.clone()
    qk = slice(0, H + Hk)
    y[:, qk, :F] = x[:, qk, :F] * cos - x[:, qk, F:R] * sin
    y[:, qk, F:R] = x[:, qk, :F] * sin + x[:, qk, F:R] * cos
    out = {"q": y[:, :H]}
    past, top = case["past"], s["max_length"]
    counts = _counts(M, case["seqs"])
    for name, which, new in (("k", 0, y[:, H:H + Hk]), ("v", 1, y[:, H + Hk:])):
        new = new.half().double()
        scales = s["cache"][3 + which].double()
        full = torch.zeros((case["seqs"], Hk, top, D), dtype=torch.float64, device="cuda")
        row = 0
        for b, n in enumerate(counts):
            end = past + n
            if past:
                full[b, :, :past] = _rows64(s["cache"], b, past, "fp8")[which]
            mine = new[row:row + n].transpose(0, 1)
            row += n
            first = past // BLOCK
            blocks = -(-end // BLOCK) - first
            # The touched blocks' slots: old rows, then the new ones, then nothing.
            rows = torch.zeros((Hk, blocks * BLOCK, D), dtype=torch.float64, device="cuda")
            lead = past - first * BLOCK
            rows[:, :lead] = full[b, :, first * BLOCK:past]
            fresh = torch.zeros_like(rows)
            fresh[:, lead:lead + n] = mine
            largest = fresh.abs().view(Hk, blocks, -1).amax(-1)
            e = torch.ceil(torch.log2((largest / 448).clamp(min=2.0 ** -15)))
            if lead:   # the first block's scale so far
                page = int(s["cache"][2][b, first * BLOCK // case["page"]])
                so_far = scales[page, :, first % (case["page"] // BLOCK)]
                e[:, 0] = torch.maximum(e[:, 0], torch.log2(so_far))
            unit = torch.exp2(e).repeat_interleave(BLOCK, 1).unsqueeze(-1)
            rows[:, lead:lead + n] = mine
            rows = _e4m3(rows / unit) * unit
            rows = torch.where(unit == 256, rows.clamp(-61440, 61440), rows)
            full[b, :, first * BLOCK:end] = rows[:, :end - first * BLOCK]
        out[name] = full
    return out


def exact(case, seed):
    if case["op"] in ("fork", "compact"):   # whole numbers and copies only
        return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend,
            "prompt": _exact_prompt}[case["op"]](case, s)
