"""rest_paged_attention where queries, keys or values are not finite: a row is what 64 bits give for the
keys that it sees, infinities and NaN included, whichever kernel shape its unit takes and whether or not
a share's border cuts it."""
import math

import numpy as np
import pytest
import torch

import paged_util as plain
import paper_2311_08252_b200 as rest
from gpu_util import to_dev
from test_gpu_paged_attention import BF16, FP16, make

pytestmark = pytest.mark.gpu


def row(c, b, r):
    """(page, row in it) of row r of context b."""
    return plain.row_of(c["table"], c["k"].shape[2], c["k"].shape[0], b, r)


def reference(c, window=0, sinks=0):
    """plain.attention; NaN and infinities of the inputs go through its 64-bit products as they are."""
    return plain.attention(c["q"], c["k"], c["v"], c["table"], c["kv_len"], c["mask"], 1 / math.sqrt(c["q"].shape[3]),
                           window, sinks, c["nodes"])


def device(c):
    args = [c[x].cuda() for x in "qkv"] + [to_dev(c["table"]), to_dev(c["kv_len"])]
    args.append(None if c["mask"] is None else to_dev(c["mask"].view(np.int32)))
    return args, None if c["nodes"] is None else to_dev(c["nodes"])


def attend(args, n_nodes, window=0, sinks=0):
    B, N, H, D = args[0].shape
    out = torch.full_like(args[0], 7.0)
    lse = torch.full((B, H, N), 5.0, device="cuda")
    rest.rest_paged_attention(*args, 1 / math.sqrt(D), window=window, sinks=sinks, n_nodes=n_nodes, out=out, lse=lse)
    return out, lse


def assert_same_kind(got, ref, live):
    """NaN, +infinity and -infinity in the same places (live: rows that exist)."""
    got, ref = got.double().cpu()[live], ref[live]
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(ref)), (kind.__name__, int(kind(got).sum()), int(kind(ref).sum()))


def exists(c):
    """Rows [B,N] of nodes that exist."""
    B, N = c["q"].shape[:2]
    nodes = np.full(B, N) if c["nodes"] is None else c["nodes"]
    return torch.from_numpy(np.arange(N)[None] < nodes[:, None])


def assert_attention(out, lse, c, ref):
    """Kinds everywhere, and paged_util.assert_attention's bounds where 64 bits are finite (columns and rows
    do not mix, so a column's bound has its own sum of magnitudes)."""
    live = exists(c)
    assert_same_kind(out, ref[0], live)
    assert_same_kind(lse.transpose(1, 2), ref[1].transpose(1, 2), live)
    finite = ref[0].isfinite() & live[:, :, None, None]
    got = torch.where(finite, out.double().cpu(), math.nan)
    want = tuple(torch.where(finite, t, math.nan) for t in (ref[0], ref[2]))
    plain.assert_attention(torch.where(got.isnan(), 0.0, got), None, (want[0], ref[1], want[1], ref[3]), c["q"].dtype,
                           int(c["kv_len"].max()) + c["q"].shape[1])


@pytest.mark.parametrize("N,G,D,few", [(40, 4, 128, 20), (66, 2, 64, 60), (140, 1, 128, 100), (128, 5, 128, 128),
                                       (150, 2, 128, 150)])
def test_values_taken_out_by_the_other_row_tile_come_back(N, G, D, few):
    """More than 128 rows by shape, but no more than 128 in this context or in its last row block: two row
    tiles take the key tiles in turn.  NaN in the V of a node in sight, in the last key tile (keys in the
    cache, values not, so that the tiles are checked late): every row that sees it is NaN, no other one."""
    B, H_kv, page = 24, 3, 64
    lens = [64 * (1 + b % 8) + (0, 63, 1, 30)[b % 4] for b in range(B)]
    c = make(N + G, B, N, G * H_kv, H_kv, D, page, lens, BF16, [few] * B)
    for b in range(B):
        at = row(c, b, lens[b] + (few - 1 if b % 2 else 0))
        c["v"][at[0], :, at[1], 5:D:7] = math.nan
    ref = reference(c)
    assert ref[0][exists(c)].isnan().any() and not ref[0][exists(c)].isnan().all()
    args, n_nodes = device(c)
    flush = torch.empty(256 << 20, dtype=torch.int8, device="cuda")
    for _ in range(4):
        flush.zero_()
        args[1].view(torch.int16).sum()
        out, lse = attend(args, n_nodes)
        assert_attention(out, lse, c, ref)


# units of 1, 24, 48, 100 rows (four, four, two copies of the rows, none), 130 rows, and 130 by shape of which
# 100 exist (two row tiles that take the key tiles in turn)
SHAPES = [(1, 1, 128, 1), (6, 4, 64, 6), (48, 1, 128, 48), (50, 2, 128, 50), (130, 1, 64, 130), (65, 2, 128, 50)]
# whole units (many contexts: a share holds several) and cut ones (one context over all blocks)
SPREADS = [([130, 64, 16, 0, 63, 300] * 30, 2), ([1500], 2)]


def small(seed, N, G, D, few, lens, H_kv, dtype=BF16):
    return make(seed, len(lens), N, G * H_kv, H_kv, D, 16, lens, dtype, [few] * len(lens))


def against_64_bits(c, window=0, sinks=0):
    """All contexts in one call; up to 14 of them against 64 bits."""
    B = len(c["kv_len"])
    some = np.sort(np.random.default_rng(B).permutation(B)[:14])
    part = {**c, **{x: c[x][some] for x in ("q", "table", "kv_len", "mask", "nodes")}}
    ref = reference(part, window, sinks)
    args, n_nodes = device(c)
    out, lse = attend(args, n_nodes, window, sinks)
    assert_attention(out[some], lse[some], part, ref)
    return ref


@pytest.mark.parametrize("lens,H_kv", SPREADS)
@pytest.mark.parametrize("N,G,D,few", SHAPES)
def test_a_query_of_nan_gives_nan(N, G, D, few, lens, H_kv):
    c = small(1, N, G, D, few, lens, H_kv)
    c["q"][:, few // 2, ::2] = math.nan
    ref = against_64_bits(c)
    assert ref[0][:, few // 2, ::2].isnan().all() and ref[0][:, few // 2, 1::2].isfinite().all()


@pytest.mark.parametrize("lens,H_kv", SPREADS)
@pytest.mark.parametrize("N,G,D,few", SHAPES)
def test_one_key_of_nan_in_sight_gives_nan(N, G, D, few, lens, H_kv):
    """In context after context another key: a prefix row (all rows see it), or a node (it and those below)."""
    c = small(2, N, G, D, few, lens, H_kv)
    for b, L in enumerate(c["kv_len"].tolist()):
        r = [L + few - 1, 0, L // 2, L - 1, L + few // 2][b % 5]
        at = row(c, b, max(r, 0))
        c["k"][at[0], b % H_kv, at[1], 3] = math.nan
    ref = against_64_bits(c)
    assert ref[0].isnan().any()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("lens,H_kv", SPREADS)
@pytest.mark.parametrize("N,G,D,few", SHAPES)
def test_infinite_values_in_sight_give_infinities(N, G, D, few, lens, H_kv, dtype):
    """V of +infinity, -infinity and NaN, alone and together, in prefix rows and nodes."""
    c = small(3, N, G, D, few, lens, H_kv, dtype)
    for b, L in enumerate(c["kv_len"].tolist()):
        for j, (r, d, x) in enumerate([(0, 1, math.inf), (L // 2, 2, -math.inf), (L - 1, 3, math.inf), (L - 1, 40, math.nan),
                                       (L + few - 1, 1, -math.inf), (L + few - 1, 4, math.inf), (L, 63, -math.inf),
                                       (L // 3, 5, math.inf), (2 * L // 3, 5, -math.inf), (2 * L // 3, 6, -math.inf)]):
            if (b + j) % 3:
                at = row(c, b, max(r, 0))
                c["v"][at[0], :, at[1], d] = x
    ref = against_64_bits(c)
    assert ref[0].isposinf().any() and ref[0].isneginf().any() and ref[0].isnan().any()
    if max(lens) > 1000:
        against_64_bits(c, window=200, sinks=20)


@pytest.mark.parametrize("N,G,D,few", SHAPES)
def test_an_infinite_value_of_tiny_weight(N, G, D, few):
    """A key whose probability rounds to nothing in the cache's type is seen all the same."""
    c = small(4, N, G, D, few, [700], 2, FP16)
    c["q"] = c["q"].abs()
    for r, x in ((3, -30.0), (500, -30.0), (699, 4.0)):
        at = row(c, 0, r)
        c["k"][at[0], :, at[1]] = x / D ** 0.5
        if x < 0:
            c["v"][at[0], :, at[1], 7 + r % 2] = math.inf
    ref = against_64_bits(c)
    assert ref[0][0, :few, :, 7:9].isposinf().all()


@pytest.mark.parametrize("G,dtype", [(2, BF16), (40, FP16), (100, BF16)])
def test_an_infinity_in_long_contexts(G, dtype):
    """Whole units of a thousand key tiles: looking for what the infinity comes to takes longer than any
    other wait, and no one gives up meanwhile (the flags are looked at behind every test)."""
    B, H_kv, D, page, L = 150, 2, 64, 256, 64000
    W = L // page + 1
    gen = torch.Generator("cuda").manual_seed(G)
    k, v = (torch.randn((B * W, H_kv, page, D), generator=gen, device="cuda", dtype=dtype) for _ in range(2))
    q = torch.randn((B, 1, G * H_kv, D), generator=gen, device="cuda", dtype=dtype)
    table = torch.randperm(B * W, generator=torch.Generator().manual_seed(1)).int().view(B, W)
    args = (q, k, v, table.cuda(), torch.full((B,), L, dtype=torch.int32, device="cuda"), None, 0.05)
    first, last = table[:, 0].long().cuda(), table[:, (L - 5) // page].long().cuda()
    for x in (first, last):
        v[x, :, (L - 5) % page, 9] = 0.0
    want = rest.rest_paged_attention(*args)
    assert want.isfinite().all()
    v[first[::2], :, (L - 5) % page, 9] = math.inf
    v[last[1::3], :, (L - 5) % page, 9] = -math.inf
    got = rest.rest_paged_attention(*args)
    rest_of = torch.arange(D, device="cuda") != 9
    assert torch.equal(got[..., rest_of], want[..., rest_of])
    for b in range(B):
        plus, minus = b % 2 == 0, b % 3 == 1
        x = got[b, 0, :, 9]
        assert (x.isnan() if plus and minus else x.isposinf() if plus else x.isneginf() if minus else x == want[b, 0, :, 9]).all(), b
