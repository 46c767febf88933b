"""Argument checks of the chunk and window calls that need no device."""
import ctypes

import pytest

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
