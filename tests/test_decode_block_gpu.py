"""The cache's operators used together, with the W4A4 layers (examples/decode_block.py)."""
import importlib.util
import os

import pytest
import torch

import paper_2409_20361_amd as rrs

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_spec = importlib.util.spec_from_file_location(
    "decode_block", os.path.join(ROOT, "examples", "decode_block.py"))
decode_block = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(decode_block)


def _block(format, **kw):
    a = dict(hidden=512, heads=8, kv_heads=2, page_size=16, prompt=40, budget=48, slack=16,
             recent=8)
    a.update(kw)
    return decode_block.AttentionBlock(3, format=format, **a)


@pytest.mark.parametrize("format", [rrs.KV_F16, rrs.KV_INT4])
def test_step_is_the_plain_computation_on_the_cached_values(format):
    block = _block(format)
    gen = torch.Generator(device="cuda").manual_seed(3)
    block.prompt(torch.randn((3, 40, 512), generator=gen, device="cuda").half())
    for i in range(60):
        x = torch.randn((3, 512), generator=gen, device="cuda").half()
        # The step's own attention, recomputed from the cache it has written.
        before, n = block.weights.clone(), block.longest + 1
        trims = n >= block.budget + block.slack
        qkv = rrs.linear(x, *block.qkv, block.group)
        q = rrs.rope_kv_append(qkv, block.positions, block.rope, block.cache, block.seq,
                               block.lengths, block.heads, weights=before)
        k, v = rrs.kv_read(block.cache, block.lengths + 1, n)
        s = q.float().view(3, 2, 4, 64) @ k.float().transpose(-1, -2) / 8.0
        p = torch.softmax(s, -1)
        o = (p @ v.float()).reshape(3, -1)
        y = block.step(x)
        if not trims:   # else the step has moved the cache
            a = rrs.paged_attention(q, block.cache, torch.full_like(block.lengths, n), n)
            # float16 output and weights: 2^-11 each, of values below max |v|
            assert (a.view(3, -1).float() - o).abs().max() <= 2.0 ** -10 * v.abs().max()
            assert torch.equal(y, rrs.linear(a.view(3, -1), *block.out, block.group))
            gain = block.weights[..., :n] - before[..., :n]
            assert (gain - p.sum(2)).abs().max() <= 1e-4
        assert torch.isfinite(y).all()


def test_the_cache_stays_within_its_budget_and_keeps_recent_tokens():
    block = _block(rrs.KV_INT4)
    gen = torch.Generator(device="cuda").manual_seed(4)
    block.prompt(torch.randn((3, 64, 512), generator=gen, device="cuda").half())
    assert block.longest == 48
    for i in range(100):
        block.step(torch.randn((3, 512), generator=gen, device="cuda").half())
        n = int(block.lengths.max())
        assert n == block.longest < block.budget + block.slack
        pos = block.slot_pos[..., :n]
        newest = int(block.positions.max()) - 1
        for t in range(max(0, newest - 7), newest + 1):   # the last 8 positions are all there
            assert (pos == t).any(-1).all()
        assert (pos.sort(-1).values.diff(dim=-1) > 0).all()   # and none is there twice


def test_main_runs():
    y = decode_block.main(["--steps", "3", "--batch", "2", "--prompt", "20", "--budget", "21"])
    assert torch.isfinite(y).all()
