"""rest_paged_attention with masks that no tree has: rows without a bit of their own, and bits of nodes that
do not exist.  A mask row of d bits stands at position kv_len + max(d, 1) - 1."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import BF16, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 0), (3, 1), (17, 60)])
@pytest.mark.parametrize("N,H,H_kv,D", [(20, 2, 2, 128), (40, 4, 1, 64), (66, 4, 2, 128)])
def test_nodes_that_others_see_and_that_see_nothing(N, H, H_kv, D, window, sinks):
    """A node without a bit stands where a child of the root does, as a row and as a key."""
    c = make(N + window, 4, N, H, H_kv, D, 16, [0, 40, 64, 129], BF16, [N, N, N - 1, N // 2])
    rng = np.random.default_rng(N)
    empty = rng.random((4, N)) < 0.4
    empty[:, 0] = True
    c["mask"][empty] = 0
    c["mask"][~empty, 0] |= np.uint32(1)           # all others see node 0, which sees nothing
    check(c, window, sinks)
