"""Calls that follow one another on a stream without a wait: each sees what the one before wrote."""
import pytest
import torch

from test_gpu_chunk import Case
from test_gpu_chunk_features import check_features

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,g,lens", [(128, 4, [100, 7]), (64, 2, [3, 260])])
def test_attention_and_features_one_after_another_on_the_same_buffers(D, g, lens):
    # One log-sum-exp buffer for all rounds: a value of the round before would be that of other queries.
    c = Case(2, g, D, [400, 150], cap=1500)
    rounds = [c.chunk(lens) for _ in range(3)]
    lse, out = torch.empty(rounds[0][2].shape[:2], device="cuda"), torch.empty_like(rounds[0][2])
    first = [c.cache.export_features(0, s) for s in range(2)]
    torch.cuda.synchronize()
    for k, v, q in rounds:
        c.cache.append_chunk_attn(0, k, v, q, lens, out=out, lse=lse)
        c.cache.chunk_features(0, q, lse, lens)
    after = [c.cache.export_features(0, s) for s in range(2)]
    # The same with a wait behind every call, each step against the definition.
    d = Case(2, g, D, [400, 150], cap=1500)
    assert all(torch.equal(d.cache.export_features(0, s), first[s]) for s in range(2))
    for k, v, q in rounds:
        torch.cuda.synchronize()
        one = torch.empty_like(lse)
        d.cache.append_chunk_attn(0, k, v, q, lens, lse=one)
        d.extend(k, v, lens)
        old = [d.cache.export_features(0, s) for s in range(2)]
        torch.cuda.synchronize()
        d.cache.chunk_features(0, q, one, lens)
        check_features(d, q, lens, old)
    for s in range(2):
        assert torch.equal(after[s], d.cache.export_features(0, s))
    assert c.status() == 0 and torch.equal(lse, one)
