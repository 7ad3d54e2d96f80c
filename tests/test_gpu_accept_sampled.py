"""rest_accept_sampled against the walk in 64 bits.  Outputs are whole numbers and have to be equal:
the seeds below put no comparison within 1e-7 of its border (weights are exact to 2^-44, or to a few
2^-53 relative where that is more, so only a closer border could fall the other way)."""
import numpy as np
import pytest
import torch

import paged_util as plain
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


def trees(rng, B, N, V, max_depth, likely=None):
    parents = np.full((B, N), -1, np.int32)
    tokens = rng.integers(0, V, (B, N)).astype(np.int32)
    for b in range(B):
        for i in range(1, N):
            parents[b, i] = rng.integers(-1, i)
    return tokens, parents


def run(logits, tokens, parents, nodes, uni, temp, top_p, depth, **kw):
    got = rest.rest_accept_sampled(logits, to_dev(tokens), to_dev(parents), to_dev(nodes), to_dev(uni), to_dev(temp),
                                   to_dev(top_p), depth, **kw)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in got]


def check(logits, tokens, parents, nodes, uni, temp, top_p, depth):
    want = plain.accept_sampled(logits.double().cpu().numpy(), tokens, parents, nodes, uni, temp, top_p, depth)
    for workspace in (None, False):                       # every row at once (few contexts), and row by row
        got = run(logits, tokens, parents, nodes, uni, temp, top_p, depth, workspace=workspace)
        for g, w in zip(got, want):
            assert np.array_equal(g, w), (g, w)
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,N,V,depth", [(1, 1, 1, 1), (4, 5, 2, 3), (30, 16, 40, 16), (9, 64, 1000, 10), (5, 256, 4097, 16),
                                         (2, 33, 32000, 5), (3, 4, 131071, 4)])
def test_matches_64_bits(B, N, V, depth, dtype):
    rng = np.random.default_rng(V + N)
    g = torch.Generator().manual_seed(V)
    tokens, parents = trees(rng, B, N, V, depth)
    logits = torch.randn((B, N + 1, V), generator=g) * 2
    for b in range(B):                                   # drafted tokens are likely ones
        for i in range(N):
            logits[b, parents[b, i] + 1, tokens[b, i]] = np.log(V) + 2 + rng.normal()
    nodes = rng.integers(0, N + 1, B).astype(np.int32)
    nodes[0] = N
    uni = rng.random((B, N + 1)).astype(np.float32)
    temp = rng.choice([0.0, 0.3, 0.8, 1.0, 2.0], B).astype(np.float32)
    top_p = rng.choice([0.1, 0.5, 0.95, 0.999, 1.0], B).astype(np.float32)
    check(logits.to(dtype).cuda(), tokens, parents, nodes, uni, temp, top_p, depth)
    check(logits.to(dtype).cuda(), tokens, parents, nodes, uni, np.full(B, 0.8, np.float32), np.full(B, 0.95, np.float32), depth)


@pytest.mark.parametrize("V", [7, 100, 5000, 40000])
def test_ties_flat_rows_and_peaked_rows(V):
    """Rows of equal logits (every token ties at the cut), of few distinct values, and of one spike."""
    rng = np.random.default_rng(V)
    B, N = 12, 6
    tokens, parents = trees(rng, B, N, V, 6)
    logits = torch.zeros((B, N + 1, V))
    logits[4:8] = torch.from_numpy(rng.integers(-3, 3, (4, N + 1, V)).astype(np.float32))
    logits[8:, :, V // 2] = 60.0
    logits[10, :, 0] = -0.0
    uni = rng.random((B, N + 1)).astype(np.float32)
    uni[:, 0] = np.linspace(0, 1, B, endpoint=False)
    check(logits.cuda(), tokens, parents, np.full(B, N, np.int32), uni, np.full(B, 1.0, np.float32),
          rng.choice([0.3, 0.7, 0.9, 1.0], B).astype(np.float32), 6)


def test_infinities_nan_and_rows_without_a_token():
    B, N, V = 8, 3, 50
    rng = np.random.default_rng(1)
    tokens, parents = trees(rng, B, N, V, 3)
    logits = torch.randn((B, N + 1, V), generator=torch.Generator().manual_seed(3))
    logits[0] = -np.inf                                   # nothing can be drawn
    logits[1, :, 10:] = -np.inf
    logits[2, :, ::2] = float("nan")
    logits[3] = float("nan")
    logits[4, :, 7] = np.inf                              # certain
    logits[5, :, [3, 9]] = np.inf                         # two certain tokens share the mass
    logits[6] = -1e30
    logits[7] = torch.linspace(-3e38, 3e38, V)
    uni = rng.random((B, N + 1)).astype(np.float32)
    for temp, p in ((1.0, 0.9), (0.7, 1.0), (0.0, 0.5)):
        got = check(logits.cuda(), tokens, parents, np.full(B, N, np.int32), uni, np.full(B, temp, np.float32),
                    np.full(B, p, np.float32), 3)
        assert got[2][0, 0] == -1 and got[2][3, 0] == -1 and got[2][4, got[0][4]] in (7,)


def test_odd_arguments():
    """Uniforms at and outside their ends, tokens outside the vocabulary, the same token twice among
    siblings, temperatures and nuclei at their ends, trees without nodes."""
    B, N, V = 10, 8, 30
    rng = np.random.default_rng(6)
    tokens, parents = trees(rng, B, N, V, 8)
    tokens[0, :4] = [-1, V, 1 << 30, -(1 << 31)]
    parents[1] = -1
    tokens[1] = [4, 4, 9, 4, 9, 9, 2, 4]
    logits = torch.randn((B, N + 1, V), generator=torch.Generator().manual_seed(5)) * 3
    uni = rng.random((B, N + 1)).astype(np.float32)
    uni[2], uni[3], uni[4], uni[5] = 0.0, 1.0, -3.0, np.nan
    uni[1, 1:] = 0.9999
    nodes = np.array([N, N, N, N, N, N, 0, -5, 99, N], np.int32)
    for temp in (1.0, 1e-30, 1e30, -1.0, np.nan):
        for p in (1.0, 2.0, 0.0, -1.0, 1e-9, 0.99999994, np.nan):
            pp = np.full(B, p, np.float32)
            check(logits.cuda(), tokens, parents, nodes, uni, np.full(B, temp, np.float32), pp, 8)


def test_strided_rows():
    B, N, V = 3, 4, 64
    rng = np.random.default_rng(2)
    tokens, parents = trees(rng, B, N, V, 4)
    wide = (torch.randn((N + 1, B, 2 * V + 1), generator=torch.Generator().manual_seed(9)) * 3).cuda()
    logits = wide.permute(1, 0, 2)[:, :, 3:3 + V]         # rows that start off any vector boundary
    uni = rng.random((B, N + 1)).astype(np.float32)
    for t in (logits, logits.bfloat16()):
        check(t, tokens, parents, np.full(B, N, np.int32), uni, np.full(B, 0.9, np.float32), np.full(B, 0.9, np.float32), 4)


def test_greedy_equals_rest_accept():
    rng = np.random.default_rng(8)
    B, N, V, depth = 20, 64, 500, 10
    tokens, parents = trees(rng, B, N, V, depth)
    logits = torch.randn((B, N + 1, V), generator=torch.Generator().manual_seed(1)).cuda()
    for b in range(B):
        for i in range(0, N, 2):
            logits[b, parents[b, i] + 1, tokens[b, i]] = 9.0 + i * 0.01
    nodes = rng.integers(0, N + 1, B).astype(np.int32)
    got = run(logits, tokens, parents, nodes, rng.random((B, N + 1)).astype(np.float32), np.zeros(B, np.float32),
              np.ones(B, np.float32), depth)
    want = rest.rest_accept(to_dev(tokens), to_dev(parents), to_dev(nodes), logits.argmax(-1).int(), depth)
    for g, w in zip(got, want):
        assert np.array_equal(g, w.cpu().numpy())


def test_emitted_tokens_follow_the_target_distribution():
    """40000 walks over one small tree: the first emitted token is distributed as the nucleus of the root's
    row, whatever the tree proposes.  Each frequency is within 5 standard deviations of p."""
    B, V = 40000, 12
    rng = np.random.default_rng(0)
    row = rng.normal(size=V) * 1.5
    logits = torch.from_numpy(np.tile(row, (B, 4, 1)).astype(np.float32)).cuda()
    order = np.argsort(-row)
    tokens = np.tile(order[[0, 3, 1]].astype(np.int32), (B, 1))
    parents = np.tile(np.array([-1, -1, 0], np.int32), (B, 1))
    uni = rng.random((B, 4)).astype(np.float32)
    got = run(logits, tokens, parents, np.full(B, 3, np.int32), uni, np.full(B, 0.8, np.float32), np.full(B, 0.9, np.float32), 2)
    w = np.exp((row - row.max()) / np.float64(np.float32(0.8)))
    before = np.cumsum(w[order]) - w[order]
    w[order[before >= np.float64(np.float32(0.9)) * w.sum()]] = 0
    p = w / w.sum()
    freq = np.bincount(got[2][:, 0], minlength=V) / B
    assert (np.abs(freq - p) <= 5 * np.sqrt(p * (1 - p) / B) + 1e-12).all()
    assert (p == 0).any() and (freq[p == 0] == 0).all() and 0 < (got[0] > 0).mean() < 1
