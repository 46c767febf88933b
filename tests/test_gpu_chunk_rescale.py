"""Chunk attention where probabilities are worked out twice: the second ones are what counts."""
import math

import pytest
import torch

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,g", [(128, 4), (64, 7)])
@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("level", [-1000.0, 150.0])
def test_first_probabilities_that_leave_the_range_are_replaced(D, g, T, level):
    """Against a reference of zero, scores around `level` are all 0 or all infinite in fp32: the first key tile of every
    item, and every later one whose scores have grown past the reference's reach, is worked out again."""
    c = Case(2, g, D, [0], cap=1200)
    n = 900
    k, v, _ = c.chunk([n])
    # <q, k> scale = level + noise in the first two thirds, then steps of 40 more: channel 0 carries the level (in powers of
    # two and few bits, so that bf16 holds it), the others noise of the keys.
    step = torch.where(torch.arange(n, device="cuda") < 600, 0, 1 + torch.arange(n, device="cuda") // 100)
    lv = level + 40.0 * step
    k[:, :, 0] = (lv / 8.0).to(torch.bfloat16)[:, None]
    q = c.rand(T, 2 * g, 0.25)
    q[:, :, 0] = 8.0
    c.cache.append_chunk(0, k[:n - T].contiguous(), v[:n - T].contiguous(), [n - T])
    c.extend(k[:n - T], v[:n - T], [n - T])
    for _ in range(10):   # (the same call again, from the same state)
        lse = torch.empty((T, 2 * g), device="cuda")
        out = c.cache.append_chunk_attn(0, k[n - T:].contiguous(), v[n - T:].contiguous(), q, [T], keep_lens=[n - T], lse=lse, scale=1.0)
    c.extend(k[n - T:], v[n - T:], [T])
    c.check_chunk(out, lse, q, [T], scale=1.0)
    assert math.isfinite(float(out.float().abs().max())) and c.status() == 0
