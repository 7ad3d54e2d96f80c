"""rest_paged_attention with masks that no tree has: rows without a bit of their own, and bits of nodes that
do not exist.  A mask row of d bits stands at position kv_len + max(d, 1) - 1."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import BF16, FP16, check, make, run

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


@pytest.mark.parametrize("window,sinks", [(64, 0), (100, 70), (10, 3)])
@pytest.mark.parametrize("N,H,H_kv,D,dtype", [(70, 2, 2, 128, BF16), (200, 1, 1, 64, FP16), (96, 4, 2, 128, BF16), (33, 4, 1, 128, BF16)])
def test_bits_of_nodes_that_do_not_exist(N, H, H_kv, D, dtype, window, sinks):
    """They name no key, but the row's position counts them: a whole key tile may be out of its window that
    all nodes of a path's length see."""
    nodes = [N // 8, 1, N // 4, 3]
    c = make(N + H, 4, N, H, H_kv, D, 16, [300, 260, 64, 190], dtype, nodes)
    bits = np.zeros((4, N, 32 * c["mask"].shape[2]), np.uint8)
    rng = np.random.default_rng(N)
    for b, n in enumerate(nodes):
        bits[b, :, n:N] = rng.random((N, N - n)) < rng.random((N, 1))
        bits[b, n - 1, n:N] = 1
    c["mask"] = c["mask"] | np.packbits(bits, axis=-1, bitorder="little").view(np.uint32)
    check(c, window, sinks)


def test_bits_behind_the_last_node_say_nothing():
    """Bits from N on of a row's last mask word."""
    for N, window, sinks in ((33, 0, 0), (33, 70, 3), (7, 4, 0), (32, 100, 0)):
        c = make(N, 3, N, 4, 2, 128, 16, [300, 64, 5], BF16)
        want = run(c, window, sinks)
        if N % 32:
            c["mask"][:, :, -1] |= np.uint32((0xFFFFFFFF << (N % 32)) & 0xFFFFFFFF)
        got = run(c, window, sinks)
        assert all(torch.equal(g, w) for g, w in zip(got, want))
