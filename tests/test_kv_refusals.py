"""No GPU: what the cache operators refuse before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2406_17276_b200 import binding, build


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


GOOD = dict(q_heads=8, kv_heads=2, head_dim=128, page=16, num_pages=100, max_pages=10, max_batch=4, max_step=65, layers=2, dtype=0)


@pytest.mark.parametrize("change", [dict(q_heads=7), dict(q_heads=0), dict(kv_heads=0), dict(page=0), dict(num_pages=0), dict(max_pages=-1), dict(max_batch=0),
                                    dict(max_step=0), dict(layers=0), dict(dtype=2)])
def test_sizes_that_mean_nothing(L, change):
    cfg = binding.KVConfig(**{**GOOD, **change})
    kv = C.c_void_p(1)
    assert L.opt_tree_kv_workspace_bytes(cfg) == 0
    assert L.opt_tree_kv_create(C.byref(kv), cfg) == binding.ERR_INVALID_ARG and not kv


@pytest.mark.parametrize("change", [dict(head_dim=96), dict(head_dim=256), dict(page=8), dict(page=48), dict(page=256), dict(max_batch=40000),
                                    dict(max_pages=1 << 28), dict(max_step=1 << 30), dict(layers=40000)])
def test_sizes_that_are_not_supported(L, change):
    cfg = binding.KVConfig(**{**GOOD, **change})
    kv = C.c_void_p(1)
    assert L.opt_tree_kv_workspace_bytes(cfg) == 0
    assert L.opt_tree_kv_create(C.byref(kv), cfg) == binding.ERR_UNSUPPORTED and not kv


def test_null_arguments(L):
    assert L.opt_tree_kv_workspace_bytes(binding.KVConfig(**GOOD)) > 0
    assert L.opt_tree_kv_workspace_bytes(None) == 0
    assert L.opt_tree_kv_create(None, binding.KVConfig(**GOOD)) == binding.ERR_INVALID_ARG
    kv = C.c_void_p(1)
    assert L.opt_tree_kv_create(C.byref(kv), None) == binding.ERR_INVALID_ARG and not kv
    assert L.opt_tree_kv_destroy(None) == binding.ERR_INVALID_ARG
    assert L.opt_tree_kv_append(None, None, 0, None, None, None, None, None, None, None) == binding.ERR_INVALID_ARG
    assert L.opt_tree_kv_attend(None, None, 0, None, None, 1.0, None, None, None) == binding.ERR_INVALID_ARG
    assert L.opt_tree_kv_compact(None, None, None, None, None, 1, 1, None, None) == binding.ERR_INVALID_ARG
    assert L.opt_tree_kv_last_device_status(None, None) == binding.ERR_INVALID_ARG
    assert L.opt_tree_kv_launch_count(None) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="the message of a machine without a device")
def test_no_fallback_without_a_device():
    with pytest.raises(RuntimeError, match="no CPU fallback"):
        binding.TreeKV(8, 2, 128, 16, 100, 10, 4, 65)


def test_cache_tensors_are_looked_at():
    k, s, t = torch.zeros((1, 3, 2, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.ones((1, 3, 2)), torch.zeros((1, 3), dtype=torch.int32)
    binding.KVCache(k, k, s, s, t)
    for bad in ((k.view(torch.uint8), k, s, s, t), (k, k[:, :2], s, s, t), (k, k, s.double(), s, t), (k, k, s, s, t.long()), (k[0], k, s, s, t),
                (k, k, s[..., :1], s, t), (k, k, s, s, t[0])):
        with pytest.raises(ValueError):
            binding.KVCache(*bad)
    step = binding.KVStep(torch.zeros(2, dtype=torch.int32), mask=torch.zeros((2, 5, 1), dtype=torch.int64))
    step.c_struct(2, 6, torch.device("cpu"))
    for B, T in ((3, 6), (2, 7), (2, 70)):
        with pytest.raises(ValueError):
            step.c_struct(B, T, torch.device("cpu"))


@pytest.mark.parametrize("change", [dict(q_heads=1, kv_heads=1, max_batch=1, max_step=(1 << 31) - 1), dict(q_heads=1, kv_heads=1, max_batch=1, max_step=(1 << 30) + 1),
                                    dict(q_heads=32767, kv_heads=1, max_batch=1, max_step=65538), dict(q_heads=2, kv_heads=2, max_batch=1, max_step=(1 << 30) - 1)])
def test_sizes_whose_sums_pass_31_bits(L, change):
    """Steps longer than any sequence, and rows that with a tile's padding no longer count in 31 bits."""
    cfg = binding.KVConfig(**{**GOOD, **change})
    kv = C.c_void_p(1)
    assert L.opt_tree_kv_workspace_bytes(cfg) == 0
    assert L.opt_tree_kv_create(C.byref(kv), cfg) == binding.ERR_UNSUPPORTED and not kv
