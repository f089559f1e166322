"""Calls whose tensors are on different GPUs are refused. On fake tensors: no GPU is needed, and no call
gets as far as a launch."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2409_20361_amd as rrs

B, HK, H, D, P, PAGES, CAP, M, R = 2, 2, 4, 128, 16, 9, 64, 3, 128
F16, F32, I32 = torch.float16, torch.float32, torch.int32

SHAPES = {
    "k": ((PAGES, HK, P, D // 2), torch.uint8), "v": ((PAGES, HK, P, D // 2), torch.uint8),
    "table": ((B, CAP // P), I32), "k_scale": ((PAGES, HK, P), F16),
    "v_scale": ((PAGES, HK, P), F16), "qkv": ((M, (H + 2 * HK) * D), F16), "positions": ((M, 1), I32),
    "rope": ((50, R), F32), "seq": ((M,), I32), "slot": ((M,), I32), "weights": ((B, HK, CAP), F32),
    "slot_pos": ((B, HK, CAP), I32), "rotated": ((M, H, D), F16), "Q": ((B, H, D), F16),
    "lengths": ((B,), I32), "mask": ((B, CAP), torch.bool), "out": ((B, H, D), F16),
    "workspace": ((1 << 20,), torch.uint8), "keep_from": ((B,), I32), "kept": ((B, HK, 8), I32),
    "new_lengths": ((B,), I32), "weights_out": ((B, HK, CAP), F32), "pos_out": ((B, HK, CAP), I32),
    "K": ((B, HK, CAP, D), F16), "V": ((B, HK, CAP, D), F16),
}
CACHE = ["k", "v", "table", "k_scale", "v_scale"]


def _append(t, cache):
    rrs.rope_kv_append(t["qkv"], t["positions"], t["rope"], cache, t["seq"], t["slot"], H,
                       weights=t["weights"], slot_pos=t["slot_pos"], out=t["rotated"])


def _attend(t, cache):
    rrs.paged_attention(t["Q"], cache, t["lengths"], mask=t["mask"], weights=t["weights"],
                        workspace=t["workspace"], out=t["out"])


def _evict(t, cache):
    rrs.kv_evict(cache, t["lengths"], t["weights"], t["slot_pos"], t["keep_from"], 8,
                 out=(t["kept"], t["new_lengths"], t["weights_out"], t["pos_out"]),
                 workspace=t["workspace"])


def _read(t, cache):
    rrs.kv_read(cache, t["lengths"], out=(t["K"], t["V"]))


CALLS = [
    (_append, "qkv", CACHE + ["positions", "rope", "seq", "slot", "weights", "slot_pos", "rotated"]),
    (_attend, "Q", CACHE + ["lengths", "mask", "weights", "workspace", "out"]),
    (_evict, "lengths", CACHE + ["weights", "slot_pos", "keep_from", "kept", "new_lengths",
                                 "weights_out", "pos_out", "workspace"]),
    (_read, "lengths", CACHE + ["K", "V"]),
]


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
@pytest.mark.parametrize("device", ["cuda:1", "cpu"])
@pytest.mark.parametrize("call,name", [(c, n) for c, _, names in CALLS for n in names])
def test_another_device(call, name, device):
    with FakeTensorMode():
        t = {n: torch.empty(shape, dtype=dtype, device=device if n == name else "cuda:0")
             for n, (shape, dtype) in SHAPES.items()}
    cache = rrs.KVCache(*(t[n] for n in CACHE))
    with pytest.raises(ValueError, match="on cuda:0"):
        call(t, cache)


@pytest.mark.parametrize("call,name", [(c, n) for c, n, _ in CALLS])
def test_not_on_a_gpu(call, name):
    with FakeTensorMode():
        t = {n: torch.empty(shape, dtype=dtype, device="cpu") for n, (shape, dtype) in SHAPES.items()}
    with pytest.raises(ValueError, match=name + " must be a GPU tensor"):
        call(t, rrs.KVCache(*(t[n] for n in CACHE)))
