"""rest_paged_attention: every key tile counts once, however long the context.  All queries are 0, so a node's
probabilities are equal, and V names the key's tile of 64 by a 1 in a column of its own: column d of a row
is the share of tile d among the keys that it sees, and a tile that is lost, doubled or read too early shows
as a whole column."""
import numpy as np
import pytest
import torch

import datagen
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 70)])
@pytest.mark.parametrize("B,N,G,H_kv,D,page,dtype,lens", [
    (1, 1, 4, 2, 128, 16, torch.bfloat16, [8000]),          # one stream: units cut into many pieces
    (1, 48, 1, 1, 128, 64, torch.bfloat16, [8100]),
    (150, 1, 4, 2, 64, 64, torch.float16, [3900, 1, 2000]),  # whole units, long ones among short ones
    (24, 12, 4, 4, 128, 16, torch.bfloat16, [2000, 7777, 300]),
    (40, 25, 4, 2, 128, 32, torch.bfloat16, [4000, 129]),     # 100 rows
    (12, 100, 2, 4, 128, 64, torch.bfloat16, [3000, 6000, 64]),
    (30, 33, 4, 4, 64, 128, torch.float16, [3900, 1234]),     # 132 rows, some contexts with 128 and fewer
    (8, 128, 5, 4, 128, 64, torch.bfloat16, [8000, 3333]),    # row blocks
])
def test_every_tile_counts_once(B, N, G, H_kv, D, page, dtype, lens, window, sinks):
    rng = np.random.default_rng(N + B)
    lens = np.array([lens[b % len(lens)] for b in range(B)], np.int32)
    nodes = np.array([N if b % 2 == 0 else max(N - 1 - b % 3, 1) for b in range(B)], np.int32)
    W = -(-(int(lens.max()) + N) // page)
    assert W * page <= 64 * (D + 1)
    table = rng.permutation(B * W).reshape(B, W).astype(np.int32)
    k = torch.randn((B * W, H_kv, page, D), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(dtype)
    tile = torch.arange(W * page, device="cuda") // 64 % D
    one = torch.nn.functional.one_hot(tile, D).to(dtype).view(W, 1, page, D)
    v = torch.empty_like(k)
    v[to_dev(table).long()] = one.expand(B, W, H_kv, page, D)
    depth, seen, words = np.zeros((B, N), np.int64), np.zeros((B, N, N), bool), []
    for b in range(B):
        _, _, mask = datagen.make_random_tree(b + N, N, 12)
        seen[b] = np.unpackbits(mask.view(np.uint8).reshape(N, -1), axis=1, bitorder="little")[:, :N]
        depth[b] = seen[b].sum(1)
        words.append(mask)
    q = torch.zeros((B, N, G * H_kv, D), dtype=dtype, device="cuda")
    args = (q, k, v, to_dev(table), to_dev(lens), to_dev(np.stack(words).view(np.int32)), 0.1)

    # the shares, from positions
    key = torch.arange(W * page, device="cuda")[None, None]
    L, n = to_dev(lens).long()[:, None, None], to_dev(nodes).long()[:, None, None]
    d, s = to_dev(depth), to_dev(seen)
    at_node = (key - L).clamp(0, N - 1)
    sees = (key < L) | ((key >= L) & (key < L + n) & s.gather(2, at_node.expand(B, N, W * page)))
    if window:
        at = torch.where(key < L, key, L + d.gather(1, at_node[:, 0])[:, None] - 1)
        sees &= (at < sinks) | (at > L + d[:, :, None] - 1 - window)
    count = torch.zeros((B, N, D), dtype=torch.float64, device="cuda")
    count.scatter_add_(2, tile.expand(B, N, -1), sees.double())
    total = sees.sum(2, keepdim=True).double()
    want = (count / total)[:, :, None].expand(B, N, G * H_kv, D)
    live = torch.arange(N, device="cuda")[None] < to_dev(nodes)[:, None]

    flush = torch.empty(256 << 20, dtype=torch.int8, device="cuda")
    lse = torch.empty((B, G * H_kv, N), device="cuda")
    for _ in range(3):
        flush.zero_()                                          # then keys in the cache, values not
        k.view(torch.int16).sum()
        out = rest.rest_paged_attention(*args, window=window, sinks=sinks, n_nodes=to_dev(nodes), lse=lse)
        # probabilities before the division are 1, their sums whole numbers: the output's rounding, and 2^-21 for
        # 1 / sum and its product
        err = ((out.double() - want).abs() / want.clamp(min=1e-30)).where(want > 0, out.double().abs())[live]
        assert err.max() <= torch.finfo(dtype).eps / 2 + 2.0 ** -21, float(err.max())
        # log of a whole number below 2^14: 2^-22 of its value for the logarithm and the product
        got = lse.transpose(1, 2)[live].double()
        assert (got - total.log()[live]).abs().max() <= 2.0 ** -22 * 10
