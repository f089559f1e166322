#!/usr/bin/env python3
"""The attention half of a decoder layer on the W4A4 library, from prompts to single tokens.

    python examples/decode_block.py [--int4] [--steps N] [--batch B] [--prompt T] [--budget C]

A fused QKV projection and an output projection (rrs.linear) with the paged key/value cache
between them: rrs.rope_kv_append writes the cache, rrs.paged_attention reads it for every new token
and accumulates the weights that each cached token receives, and rrs.kv_evict brings the cache
back to its budget whenever it has outgrown it. Random weights of the LLaMA-7B shape
(hidden size 4096, 32 heads of 128; here with 8 KV heads), random tokens.
"""
import argparse
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2409_20361_amd as rrs  # noqa: E402


def _weight(K, N, gen):
    return rrs.prepare_weight((0.02 * torch.randn((K, N), generator=gen, device="cuda")).half())


class AttentionBlock:
    """batch sequences with a cache of at most budget + slack tokens each."""

    def __init__(self, batch, hidden=4096, heads=32, kv_heads=8, group=128, page_size=64,
                 prompt=512, budget=1024, slack=64, recent=32, format=rrs.KV_F16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.batch, self.hidden, self.heads, self.group = batch, hidden, heads, group
        self.budget, self.slack, self.recent = budget, slack, recent
        self.dim = hidden // heads
        self.qkv = _weight(hidden, (heads + 2 * kv_heads) * self.dim, gen)
        self.out = _weight(hidden, hidden, gen)
        top = max(prompt, budget + slack)
        per_seq = -(-top // page_size)
        table = torch.randperm(batch * per_seq, generator=gen, device="cuda")
        self.cache = rrs.kv_cache(batch * per_seq, kv_heads, page_size, self.dim,
                                  table.to(torch.int32).view(batch, per_seq), format)
        self.rope = rrs.rope_table(1 << 16, self.dim)
        slots = (batch, kv_heads, self.cache.capacity)
        self.weights = torch.zeros(slots, device="cuda")
        self.slot_pos = torch.full(slots, -1, dtype=torch.int32, device="cuda")
        self.seq = torch.arange(batch, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.positions = torch.zeros((batch, 1), dtype=torch.int32, device="cuda")
        self.longest = 0   # what the host knows of the lengths
        self.workspace = torch.zeros(   # of the linear layers, for every call
            max(rrs.linear_workspace_bytes(batch * n, hidden, group) for n in (1, top)),
            dtype=torch.uint8, device="cuda")

    def _linear(self, x, weight):
        return rrs.linear(x, *weight, self.group, workspace=self.workspace)

    def _append(self, x, positions, seq, slot):
        qkv = self._linear(x, self.qkv)
        return rrs.rope_kv_append(qkv, positions, self.rope, self.cache, seq, slot, self.heads,
                                  weights=self.weights, slot_pos=self.slot_pos)

    def prompt(self, x):
        """x: (batch, T, hidden) fp16. Causal attention over the prompt in plain torch, from the cached
        values, as later tokens will see them."""
        B, T, _ = x.shape
        slot = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B)
        q = self._append(x.reshape(B * T, -1), slot.view(-1, 1),
                         self.seq.repeat_interleave(T), slot)
        self.lengths.fill_(T)
        self.positions.fill_(T)
        self.longest = T
        k, v = rrs.kv_read(self.cache, self.lengths, T)
        group = self.heads // k.shape[1]
        q = q.view(B, T, -1, group, self.dim).permute(0, 2, 3, 1, 4).float()
        s = q @ k.float().transpose(-1, -2).unsqueeze(2) * self.dim ** -0.5
        later = torch.ones((T, T), dtype=torch.bool, device="cuda").triu(1)
        p = torch.softmax(s.masked_fill(later, float("-inf")), -1)
        self.weights[..., :T] += p.sum((2, 3))
        y = (p @ v.float().unsqueeze(2)).permute(0, 3, 1, 2, 4).reshape(B * T, -1).half()
        y = self._linear(y, self.out).view(B, T, -1)
        self.trim()
        return y

    def step(self, x):
        """One new token per sequence: x (batch, hidden) fp16 -> (batch, hidden)."""
        q = self._append(x, self.positions, self.seq, self.lengths)
        self.lengths += 1
        self.positions += 1
        self.longest += 1
        y = rrs.paged_attention(q, self.cache, self.lengths, max_length=self.longest,
                                weights=self.weights)
        y = self._linear(y.view(self.batch, -1), self.out)
        if self.longest >= self.budget + self.slack:
            self.trim()
        return y

    def trim(self):
        if self.longest <= self.budget:
            return
        keep_from = self.positions[:, 0] - self.recent
        _, self.lengths, self.weights, self.slot_pos = rrs.kv_evict(
            self.cache, self.lengths, self.weights, self.slot_pos, keep_from, self.budget,
            max_length=self.longest)
        self.longest = self.budget


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--int4", action="store_true", help="4-bit cache")
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--budget", type=int, default=512)
    args = ap.parse_args(argv)
    block = AttentionBlock(args.batch, prompt=args.prompt, budget=args.budget,
                           format=rrs.KV_INT4 if args.int4 else rrs.KV_F16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((args.batch, args.prompt, block.hidden), generator=gen, device="cuda").half()
    y = block.prompt(x)[:, -1]
    for i in range(args.steps + 3):
        if i == 3:
            torch.cuda.synchronize()
            began = time.perf_counter()
        y = block.step(torch.nn.functional.normalize(y.float(), dim=-1).mul_(64.0).half())
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / args.steps * 1e6
    print(f"{args.batch} sequences, {'INT4' if args.int4 else 'float16'} cache of "
          f"{block.longest} tokens (budget {args.budget}): {us:.1f} us per step")
    return y


if __name__ == "__main__":
    main()
