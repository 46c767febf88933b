"""Acceptance where a cluster's CTAs have next to nothing to read before they write to one another: the smallest vocabularies."""
import pytest
import torch

from test_gpu_verify import handle, problem, run, want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 2, 7, 256, 257, 513])
@pytest.mark.parametrize("sampled", [True, False])
def test_small_vocabularies_in_clusters_of_eight(vocab, sampled):
    """Fewer pieces than CTAs: most of them have nothing to sum, and all of them exchange what they have at once."""
    for batch in (1, 5, 37):
        x = problem([1 + s % 4 for s in range(batch)], vocab, 3, sampled, torch.float32, vocab + batch, noise=2.0)
        cache = handle(batch)
        first = run(x, cache)
        assert first == (want(x), 0)
        for _ in range(50):   # back to back: a launch's CTAs start while those of the one before still run
            got = cache.verify_tree(x["tokens"], x["parents"], x["lens"], x["target"], x["u"], x["us"], draft=x["draft"])
        assert [t.cpu().tolist() for t in got] == first[0] and cache.device_status()[0] == 0
