"""Integers past 32 bits are refused by the binding of the chunk and window calls, not cut off."""
import pytest
import torch

from paper_2602_03203_b200 import binding

BIG = (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32)


@pytest.fixture
def cache(monkeypatch):
    """A handle that no library call has made: every call here has to end ahead of the library."""
    c = binding.Cache.__new__(binding.Cache)
    c._h, c.feat_dim = None, 12
    c.cfg = binding.FkvConfig(1, 2, 2, 64, 3, 16, 16, 0, 32, 0, 64, 0, 0)
    c.workspace = torch.empty(1, dtype=torch.uint8, device="meta")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: c.workspace.device.index)
    return c


@pytest.mark.parametrize("big", BIG)
def test_lists_of_lengths(big):
    for lens in ([1, big, 2], [big, 0, 0], [0, 0, big]):
        with pytest.raises(ValueError, match="keep_lens: .* 32 bits"):
            binding._lens(lens, 3, "keep_lens")
    assert list(binding._lens([2 ** 31 - 1, 0, -2 ** 31], 3, "x")) == [2 ** 31 - 1, 0, -2 ** 31]
    with pytest.raises(TypeError):
        binding._lens([1.5, 0, 0], 3, "x")


@pytest.mark.parametrize("big", BIG)
@pytest.mark.parametrize("name", ["layer", "window", "sinks"])
def test_windows_sinks_and_layers(cache, big, name):
    t = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="meta")  # noqa: E731
    k, q, lse, lens = t(3, 2, 64), t(3, 4, 64), t(3, 4, dtype=torch.float32), [1, 2, 0]
    x = {**dict(layer=0, window=4, sinks=1), name: big}
    calls = [lambda: cache.decode_attn_window(x["layer"], q, x["window"], x["sinks"]),
             lambda: cache.append_decode_attn_window(x["layer"], k, k, q, x["window"], x["sinks"]),
             lambda: cache.chunk_attn(x["layer"], q, lens, x["window"], x["sinks"]),
             lambda: cache.append_chunk_attn(x["layer"], k, k, q, lens, window=x["window"], sinks=x["sinks"]),
             lambda: cache.chunk_features(x["layer"], q, lse, lens, x["window"], x["sinks"])]
    if name == "layer":
        calls += [lambda: cache.append_chunk(x["layer"], k, k, lens), lambda: cache.export_features(x["layer"], 0)]
    for call in calls:
        with pytest.raises(ValueError, match=f"{name}: .* 32 bits"):
            call()
