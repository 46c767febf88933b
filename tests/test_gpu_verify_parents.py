"""Parents that are none, far outside 16 bits among them: a node with one is reached from nowhere."""
import pytest
import torch

from paper_2602_03203_b200 import binding
from test_gpu_verify import handle, small

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-2, -32768, -32769, -65536, -65535, -131072, -2 ** 31, 1, 2 ** 16, 2 ** 31 - 1])
def test_bad_parents(bad):
    """Node 1 has a parent that is none, and the token that the target wants after nodes 0 and 1."""
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = handle(1)
    got = cache.verify_tree_greedy(i32(0, 5, 5, 5), i32(-1, bad, 0, bad), [4], i32(5, 5, 5, 7))
    assert [x.tolist() for x in got] == [[[0, 2, -1, -1]], [2], [[5, 5, -1, -1]]]   # (1 is a parent of node 3, but is not reached itself)
    assert cache.device_status()[0] == binding.DEV_BAD_INDEX
    p = [[0.0, 1.0]] * 4
    path, n, out, status = small([-1, bad, 0, bad], [0, 1, 1, 1], p, p, [0, 0.1, 0.1, 0.1])
    assert (path, n, out, status) == ([0, 2, -1, -1], 2, [1, 1, -1, -1], binding.DEV_BAD_INDEX)
    masks = cache.tree_masks(i32(-1, bad, 0, bad), [4]).tolist()
    assert [m[0] for m in masks] == [1, 2, 5, 10 if bad == 1 else 8] and cache.device_status()[0] == binding.DEV_BAD_INDEX
