"""Argument checks of the chunk and window calls that need no device."""
import ctypes

import pytest
import torch

from paper_2602_03203_b200 import binding


def test_null_handles_are_refused():
    lib = binding.lib()
    lens = (ctypes.c_int32 * 1)(1)
    assert lib.fkv_append_chunk(None, 0, None, None, None, None, lens, None) == -1
    assert lib.fkv_chunk_attn(None, 0, None, lens, 0, 0, 0.0, None, None, None) == -1
    assert lib.fkv_append_chunk_attn(None, 0, None, None, None, None, lens, None, 0, 0, 0.0, None, None, None) == -1
    assert lib.fkv_decode_attn_window(None, 0, None, None, 4, 0, None, 0.0, None) == -1
    assert lib.fkv_append_decode_attn_window(None, 0, None, None, None, None, None, 4, 0, None, 0.0, None) == -1
    assert lib.fkv_export_features(None, 0, 0, None, None) == -1


def test_length_lists_have_one_entry_per_sequence():
    assert binding._lens(None, 3, "x") is None
    assert list(binding._lens([1, 0, 2], 3, "x")) == [1, 0, 2]
    with pytest.raises(ValueError):
        binding._lens([1, 2], 3, "x")


def test_null_handle_of_the_features_is_refused():
    lens = (ctypes.c_int32 * 1)(1)
    assert binding.lib().fkv_chunk_features(None, 0, None, None, lens, 0, 0, 0.0, None) == -1


def test_tensors_of_another_size_or_device_are_refused(monkeypatch):
    """What the binding checks ahead of a launch; tensors without memory stand in for those of a device."""
    cache = binding.Cache.__new__(binding.Cache)
    cache._h, cache.feat_dim = None, 12
    cache.cfg = binding.FkvConfig(1, 2, 2, 64, 3, 16, 16, 0, 32, 0, 64, 0, 0)
    cache.workspace = torch.empty(1, dtype=torch.uint8, device="meta")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: cache.workspace.device.index)
    t = lambda *s, dtype=torch.bfloat16, device="meta": torch.empty(s, dtype=dtype, device=device)  # noqa: E731
    k, q, pos = t(3, 2, 64), t(3, 4, 64), t(3, dtype=torch.int32)
    cache._check_step(k, k, q, q, pos)
    cache._check_step(None, None, q, q, None)
    for bad in [(t(2, 2, 64), k, q, q, pos), (k, t(3, 2, 63), q, q, pos), (k, k, k, q, pos), (k, k, q, t(4, 4, 64), pos),
                (k, k, q, q, t(2, dtype=torch.int32)), (k, k, q, q, t(3, dtype=torch.int32, device="cpu")),
                (t(3, 2, 64, device="cpu"), k, q, q, pos)]:
        with pytest.raises(ValueError):
            cache._check_step(*bad)
    cache._check_chunk([1, 2, 0], k=k, q=q, lse=t(3, 4, dtype=torch.float32), pos=pos)
    with pytest.raises(ValueError):
        cache._check_chunk([1, 2, 0], k=k, q=t(3, 4, 64, device="cpu"))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError):
        cache._check_place(k)
