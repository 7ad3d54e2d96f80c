"""rest_paged_attention against 64 bits (bounds: see paged_util.assert_attention)."""
import math

import numpy as np
import pytest
import torch

import datagen
import paged_util as plain
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def make(seed, B, N, H, H_kv, D, page, kv_len, dtype=BF16, nodes=None, layout="hnd", spare=2, max_depth=9, tree=True):
    """Inputs on the CPU; pages in random order, the rest of the pool NaN."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    kv_len = np.asarray(kv_len, np.int32)
    W = -(-(int(kv_len.max()) + N) // page)
    P = B * W + spare
    table = rng.permutation(P)[:B * W].reshape(B, W).astype(np.int32)
    k, v = (torch.randn((P, H_kv, page, D), generator=g).to(dtype) for _ in range(2))
    used = torch.zeros((P, page), dtype=torch.bool)
    for b in range(B):
        for r in range(int(kv_len[b]) + (N if nodes is None else int(nodes[b]))):
            used[table[b, r // page], r % page] = True
    for t in (k, v):
        t.permute(0, 2, 1, 3)[~used] = float("nan")
    q = torch.randn((B, N, H, D), generator=g) * torch.linspace(0.5, 2, H)[None, None, :, None]
    mask = np.stack([datagen.make_random_tree(seed * 100 + b, N, max_depth)[2] for b in range(B)]) if tree else None
    return dict(q=q.to(dtype), k=k, v=v, table=table, kv_len=kv_len, mask=mask,
                nodes=None if nodes is None else np.asarray(nodes, np.int32), layout=layout)


def run(c, window=0, sinks=0, scale=None, want_lse=True, stream=None, workspace=None):
    D = c["q"].shape[3]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    q, k, v = c["q"].cuda(), c["k"].cuda(), c["v"].cuda()
    if c["layout"] == "nhd":                       # rows before heads in the pages, heads before rows in q and out
        k, v = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (k, v))
        q = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    out = torch.full_like(q, 7.0)
    B, N, H, _ = q.shape
    lse = torch.full((B, H, N), 5.0, device="cuda") if want_lse else None
    rest.rest_paged_attention(q, k, v, to_dev(c["table"]), to_dev(c["kv_len"]),
                              None if c["mask"] is None else to_dev(c["mask"].view(np.int32)), scale, window=window,
                              sinks=sinks, n_nodes=None if c["nodes"] is None else to_dev(c["nodes"]), out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def check(c, window=0, sinks=0, scale=None):
    D = c["q"].shape[3]
    out, lse = run(c, window, sinks, scale)
    ref = plain.attention(c["q"], c["k"], c["v"], c["table"], c["kv_len"], c["mask"],
                          1.0 / math.sqrt(D) if scale is None else scale, window, sinks, c["nodes"])
    plain.assert_attention(out, lse, ref, c["q"].dtype, int(c["kv_len"].max()) + c["q"].shape[1])
    gone = ref[0].isnan().cpu()                    # nodes that do not exist: left as they were
    assert (out.cpu()[gone] == 7.0).all() and (lse.cpu()[ref[1].isnan()] == 5.0).all()
    return out, lse, ref


@pytest.mark.parametrize("B,N,H,H_kv,D,page,L,dtype", [
    (1, 1, 1, 1, 128, 16, 0, BF16),          # one token, nothing before it
    (1, 1, 4, 1, 64, 16, 1, FP16),
    (3, 1, 32, 8, 128, 16, 200, BF16),       # ordinary decoding
    (2, 1, 8, 8, 64, 128, 1000, BF16),
    (1, 1, 8, 1, 128, 32, 2500, FP16),       # one KV head over many SMs
    (2, 64, 4, 4, 128, 64, 130, BF16),       # a tree, one KV head per head
    (2, 64, 8, 2, 128, 16, 300, BF16),       # 256 rows a KV head
    (1, 33, 10, 2, 64, 32, 77, FP16),        # five heads a KV head: 165 rows
    (2, 13, 6, 2, 128, 256, 513, BF16),
    (1, 128, 10, 2, 128, 64, 260, BF16),     # 640 rows a KV head
    (1, 256, 3, 1, 64, 16, 100, BF16),       # 768 rows
    (1, 256, 1, 1, 128, 128, 0, FP16),       # only the tree
    (5, 7, 3, 3, 64, 16, 64, BF16),
    (1, 129, 1, 1, 128, 16, 63, BF16),       # one row more than a tile
    (9, 2, 16, 4, 128, 16, 31, FP16),
])
def test_matches_64_bits(B, N, H, H_kv, D, page, L, dtype):
    check(make(B + N, B, N, H, H_kv, D, page, [L] * B, dtype))


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (1, 0), (5, 70), (3, 1)])
@pytest.mark.parametrize("N,H,H_kv,D,page", [(17, 8, 2, 128, 16), (70, 4, 1, 64, 64), (1, 6, 2, 128, 32), (150, 2, 2, 128, 16)])
def test_ragged_batches_windows_and_sinks(N, H, H_kv, D, page, window, sinks, layout):
    lens = [300, 0, 1, 129, 64, 257]
    rng = np.random.default_rng(N)
    nodes = rng.integers(0, N + 1, len(lens))
    nodes[:3] = N, max(N - 1, 1), 1
    check(make(N, len(lens), N, H, H_kv, D, page, lens, BF16, nodes, layout), window, sinks)


@pytest.mark.parametrize("D,N,dtype", [(128, 5, BF16), (64, 1, FP16), (128, 70, FP16)])
def test_pages_behind_the_window_may_be_gone(D, N, dtype):
    c = make(3, 3, N, 4, 2, D, 16, [700, 333, 90], dtype)
    window, sinks = 64, 20
    for b, L in enumerate(c["kv_len"]):
        for col in range(c["table"].shape[1]):
            if col * 16 >= sinks and (col + 1) * 16 - 1 <= L - window:
                c["k"][c["table"][b, col]] = c["v"][c["table"][b, col]] = float("nan")
                c["table"][b, col] = -1 if col % 2 else 12345     # gone, or whatever was left in the entry
    check(c, window, sinks)


@pytest.mark.parametrize("N,H,D", [(6, 2, 128), (40, 8, 64), (90, 4, 128)])
def test_a_run_of_tokens_without_a_mask(N, H, D):
    for window, sinks in ((0, 0), (16, 2)):
        check(make(N, 2, N, H, 2, D, 32, [100, 3], tree=False), window, sinks)


@pytest.mark.parametrize("N,H,H_kv", [(20, 2, 2), (64, 8, 2), (3, 1, 1)])
def test_rows_that_see_nothing(N, H, H_kv):
    c = make(5, 3, N, H, H_kv, 128, 16, [0, 40, 0])
    c["mask"][:, ::2] = 0
    out, lse, ref = check(c)
    assert (out[0, ::2] == 0).all() and torch.isneginf(lse[0, :, ::2]).all()
    c["mask"][:] = 0                                # a window of one position: a row without its own bit
    check(c, window=1)


@pytest.mark.parametrize("N,H,H_kv,D", [(24, 2, 1, 128), (64, 4, 1, 64), (130, 2, 2, 128)])
def test_what_is_masked_may_hold_anything(N, H, H_kv, D):
    """Infinities and NaN in a node's K or V reach that node and its descendants only; in rows behind
    the window they reach nobody."""
    c = make(8, 2, N, H, H_kv, D, 16, [150, 90])
    clean = {**c, "k": c["k"].clone(), "v": c["v"].clone()}
    bad = {0: (2, "v", math.nan), 1: (N // 2, "k", math.inf)}
    window, sinks = 40, 3
    for b, (node, which, value) in bad.items():
        for r in [int(c["kv_len"][b]) + node] + list(range(sinks, int(c["kv_len"][b]) - window)):
            p, at = plain.row_of(c["table"], 16, c["k"].shape[0], b, r)
            c[which][p, :, at, 3:9] = value
            clean[which][p, :, at, 3:9] = 0
    out, lse = run(c, window, sinks)
    ref = plain.attention(clean["q"], clean["k"], clean["v"], c["table"], c["kv_len"], c["mask"], 1 / math.sqrt(D),
                          window, sinks)
    for b, (node, which, _) in bad.items():
        hit = ((c["mask"][b, :, node >> 5] >> (node & 31)) & 1).astype(bool)
        assert hit.any() and not hit.all()
        got = out[b].float().cpu()
        assert not got[hit][..., 3:9].isfinite().any() if which == "v" else not got[hit].isfinite().all()
        if which == "v":
            assert got[hit][..., 9:].isfinite().all()
        for t in (ref[0], ref[2]):
            t[b, torch.from_numpy(hit)] = float("nan")
        ref[1][b, :, torch.from_numpy(hit)] = float("nan")
    plain.assert_attention(out, lse, ref, BF16, 400)


@pytest.mark.parametrize("N,D,H_kv", [(2, 128, 1), (64, 128, 1), (70, 64, 2), (130, 128, 2)])
def test_scores_whose_maximum_keeps_growing(N, D, H_kv):
    c = make(31, 2, N, 2, H_kv, D, 64, [700, 650])
    for b in range(2):
        for r in range(int(c["kv_len"][b]) + N):
            p, at = plain.row_of(c["table"], 64, c["k"].shape[0], b, r)
            c["k"][p, :, at] = (c["k"][p, :, at].float() * (1 + 7 * r / 700) * (2.5 if (r // 64) % 5 == 3 else 1)).to(BF16)
    check(c)
    check(c, window=150, sinks=70)


def test_pools_beyond_32_bit_offsets():
    B, N, H, H_kv, D, page = 2, 4, 8, 8, 128, 128
    P = (1 << 31) // (H_kv * page * D) + 40
    c = make(12, B, N, H, H_kv, D, page, [300, 500])
    W, small = c["table"].shape[1], c["k"]
    far = {int(p): P - 1 - i for i, p in enumerate(sorted(set(c["table"].ravel().tolist())))}
    k, v = (torch.zeros((P, H_kv, page, D), dtype=BF16, device="cuda") for _ in range(2))
    for p, z in far.items():
        k[z], v[z] = c["k"][p].cuda(), c["v"][p].cuda()
    assert min(far.values()) * H_kv * page * D > 1 << 31 and W * B == len(far) and small.shape[0] < P
    table = np.vectorize(far.get)(c["table"]).astype(np.int32)
    out = rest.rest_paged_attention(c["q"].cuda(), k, v, to_dev(table), to_dev(c["kv_len"]),
                                    to_dev(c["mask"].view(np.int32)), 1 / math.sqrt(D))
    ref = plain.attention(c["q"], c["k"], c["v"], c["table"], c["kv_len"], c["mask"], 1 / math.sqrt(D))
    plain.assert_attention(out, None, ref, BF16, 600)


def test_other_streams_captures_and_shared_scratch():
    """Calls on a side stream, and a captured step replayed on new inputs while an eager call of
    another shape runs in between with its own scratch: the same bits as plain calls."""
    a, b = make(1, 2, 20, 4, 1, 128, 16, [400, 90]), make(2, 1, 3, 2, 2, 128, 16, [900])
    want_a, want_b = run(a), run(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(a)
    assert torch.equal(got[0], want_a[0]) and torch.equal(got[1], want_a[1])
    q, k, v = a["q"].cuda(), a["k"].cuda(), a["v"].cuda()
    args = [to_dev(a["table"]), to_dev(a["kv_len"]), to_dev(a["mask"].view(np.int32)), 1 / math.sqrt(128)]
    out, lse = torch.zeros_like(q), torch.zeros((2, 4, 20), device="cuda")
    need = rest.paged_attention_workspace_bytes(2, 4, 1, 20, 128)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rest.rest_paged_attention(q, k, v, *args, out=out, lse=lse, workspace=ws)
    keep = q.clone()
    for _ in range(3):
        q.copy_(keep * 0.5)
        graph.replay()
        got = run(b)
        assert torch.equal(got[0], want_b[0])
        q.copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_a[0]) and torch.equal(lse, want_a[1])


def test_many_short_contexts():
    lens = np.random.default_rng(2).integers(0, 40, 700)
    check(make(44, 700, 1, 2, 1, 64, 16, lens, FP16))
    check(make(45, 300, 3, 2, 2, 128, 16, lens[:300]), window=8, sinks=2)


def test_agrees_with_the_contiguous_call_on_the_same_rows():
    B, N, H, D, L = 2, 64, 8, 128, 500
    c = make(77, B, N, H, H, D, 64, [L] * B)
    rows = torch.zeros((B, H, L + N, D), dtype=BF16), torch.zeros((B, H, L + N, D), dtype=BF16)
    for b in range(B):
        for r in range(L + N):
            p, at = plain.row_of(c["table"], 64, c["k"].shape[0], b, r)
            rows[0][b, :, r], rows[1][b, :, r] = c["k"][p, :, at], c["v"][p, :, at]
    a = rest.rest_tree_attention(c["q"].cuda(), rows[0].cuda(), rows[1].cuda(), to_dev(c["kv_len"]),
                                 to_dev(c["mask"].view(np.int32)), 1 / math.sqrt(D))
    out, _ = run(c)
    # each is within 2^-8 (|out| + A) + 2^-15 (S + 1) A of 64 bits; |out| <= A < 1 and S < 16 here
    assert (a.float() - out.float()).abs().max() <= 2 * (2 * 2.0 ** -8 + 17 * 2.0 ** -15)


@pytest.mark.parametrize("N,D,window", [(66, 128, 0), (66, 128, 150), (66, 64, 0), (40, 128, 0), (4, 128, 0)])
def test_values_that_arrive_late(N, D, window):
    """Keys in the cache, values not: the last two products of a piece are both under way at its end."""
    B, H, H_kv, page = 30, 8, 4, 64
    nodes = [N if b % 3 else N // 2 for b in range(B)]
    c = make(N + D, B, N, H, H_kv, D, page, [150 + 37 * (b % 7) for b in range(B)], BF16, nodes)
    c["q"] = (c["q"].float() * 2).to(BF16)         # peaked rows: a tile that is left out shows
    ref = plain.attention(c["q"], c["k"], c["v"], c["table"], c["kv_len"], c["mask"], 1 / math.sqrt(D), window, 0, c["nodes"])
    q, k, v = (c[x].cuda() for x in "qkv")
    table, kv_len, n, mask = (to_dev(x) for x in (c["table"], c["kv_len"], c["nodes"], c["mask"].view(np.int32)))
    flush = torch.empty(256 << 20, dtype=torch.int8, device="cuda")
    for _ in range(6):
        out = torch.full_like(q, 7.0)
        lse = torch.full((B, H, N), 5.0, device="cuda")
        flush.zero_()
        k.view(torch.int16).sum()
        rest.rest_paged_attention(q, k, v, table, kv_len, mask, 1 / math.sqrt(D), window=window, n_nodes=n, out=out, lse=lse)
        plain.assert_attention(out, lse, ref, BF16, int(c["kv_len"].max()) + N)


@pytest.mark.parametrize("N,G,D", [(128, 5, 128), (128, 5, 64), (150, 2, 128), (200, 4, 128)])
def test_row_blocks_with_shares_of_their_own(N, G, D):
    """Several row blocks, the last one lower; contexts whose nodes leave it, or all but the first one, empty."""
    lens = [700, 0, 65, 1300, 333, 4, 64, 900]
    nodes = [N, 1, N // 2, N - 1, 0, N, 64 // G, N // 3]
    check(make(N + G, len(lens), N, 2 * G, 2, D, 32, lens, BF16, nodes))
    check(make(N - G, 1, N, 2 * G, 2, D, 32, lens[:1], BF16), 100, 3)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
@pytest.mark.parametrize("N,G,H_kv,D,B", [(64, 4, 2, 128, 40), (140, 1, 3, 64, 40), (33, 4, 8, 128, 9), (64, 4, 1, 128, 3)])
def test_contexts_of_one_and_two_row_tiles_in_turn(N, G, H_kv, D, B, window, sinks):
    """Key tiles of contexts with few and with many rows cost differently; shares may begin inside one."""
    rng = np.random.default_rng(N + B)
    nodes = [int(rng.choice([0, 1, N // 3, N // 2, N - 1, N])) for _ in range(B)]
    lens = [int(rng.choice([0, 1, 64, 63, 200, 391])) for _ in range(B)]
    check(make(N + B, B, N, G * H_kv, H_kv, D, 16, lens, BF16, nodes), window, sinks)


@pytest.mark.parametrize("handle", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(handle):
    """out is cleared on the call's stream: work that waits on the current one does not wipe the result."""
    c = make(5, 2, 8, 4, 2, 128, 16, [100, 40], BF16, [8, 5])
    want, _ = run(c, want_lse=False)
    q, k, v = (c[x].cuda() for x in "qkv")
    table, kv_len, n, mask = (to_dev(x) for x in (c["table"], c["kv_len"], c["nodes"], c["mask"].view(np.int32)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                 # the current stream is busy
    out = rest.rest_paged_attention(q, k, v, table, kv_len, mask, 1 / math.sqrt(128), n_nodes=n,
                                    stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    x, y = out.cpu(), want.cpu()
    assert (x[0] == y[0]).all() and (x[1, :5] == y[1, :5]).all() and (x[1, 5:] == 0).all()
