"""More layers than a launch's second dimension holds: calls that serve all layers at once."""
import pytest
import torch

from paper_2602_03203_b200 import binding

pytestmark = pytest.mark.gpu

LAYERS, D = 65537, 64
SOME = [0, 1, 65534, 65535, 65536]


def test_fork_with_decode_queries_on_record():
    """Two caches, the places of one swapped: pairs and the features that the recorded queries give agree."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    caches = [binding.Cache(LAYERS, 1, 1, D, 2, 16, 32, num_pages=400, feature_window=8) for _ in range(2)]
    for layer in SOME:
        k, v = rand(23, 1, D), rand(23, 1, D)
        for cache in caches:
            cache.append_chunk(layer, k, v, [12, 11])
        for _ in range(3):
            k, v, q = rand(2, 1, D), rand(2, 1, D), rand(2, 1, D)
            for cache in caches:
                cache.append_decode_attn(layer, k, v, q)
    caches[1].fork([1, 0])
    assert [caches[1].lengths(i) for i in SOME] == [[14, 15]] * len(SOME)
    for cache in caches:
        cache.sync_lengths()
        for layer in SOME:
            cache.update_features(layer)
    for layer in SOME:
        assert caches[0].lengths(layer) == [15, 14] and caches[1].lengths(layer) == [14, 15]
        for s in range(2):
            for x, y in zip(caches[0].export_head(layer, s, 0), caches[1].export_head(layer, 1 - s, 0)):
                assert torch.equal(x, y) and bool(x.any())
    assert [c.device_status()[0] for c in caches] == [0, 0]


def test_commit_of_all_layers():
    cache = binding.Cache(LAYERS, 1, 1, D, 1, 16, 16, num_pages=LAYERS)
    gen = torch.Generator(device="cuda").manual_seed(2)
    k = torch.randn((LAYERS + 4, 1, D), generator=gen, device="cuda").to(torch.bfloat16)
    masks = cache.tree_masks(torch.tensor([-1, 0, 0, 1, 2], dtype=torch.int32, device="cuda"), [5])
    for layer in range(LAYERS):
        cache.append_tree(layer, k[layer:layer + 5], k[layer:layer + 5], [5], masks)
    cache.commit_tree([5], torch.tensor([[0, 2, 4]], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"))
    cache.sync_lengths()
    assert cache.device_status() == (0, 0)
    for layer in SOME + list(range(100, LAYERS, 4999)):
        assert cache.lengths(layer) == [3]
        x, _, _, pos = cache.export_head(layer, 0, 0)
        assert torch.equal(x, k[layer:layer + 5:2, 0]) and pos.tolist() == [0, 1, 2]
