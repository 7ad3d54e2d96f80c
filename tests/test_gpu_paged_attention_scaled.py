"""rest_paged_attention_scaled against 64 bits of what the codes stand for.

Bounds: the output's rounding e |out| with e half a step of its type (2^-8 bf16, 2^-11 fp16); probabilities are rounded to
fp16, 2^-11 of each; with a shift that leaves the largest of a row 2^6 at least, fp16's smallest half step, 2^-25, is 2^-31 of
the largest p * scale, of each key, times a code of 448 at most; scores, scales, sums and exponentials in 32 bits: 2^-16 (S + 1)
of each probability and of their sum (see paged_util.assert_attention)."""
import math

import numpy as np
import pytest
import torch

import datagen
import paged_util as plain
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu
BF16, FP16, F8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def make(seed, B, N, H, H_kv, D, page, kv_len, dtype=BF16, nodes=None, layout="hnd", spare=2, tree=True, spread=1, powers=True):
    """Inputs on the CPU: codes that use their range, scales of their own for each block; pages in random order, codes and
    scales of the rest of the pool NaN."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    kv_len = np.asarray(kv_len, np.int32)
    W = -(-(int(kv_len.max()) + N) // page)
    P = B * W + spare
    table = rng.permutation(P)[:B * W].reshape(B, W).astype(np.int32)
    k, v = ((torch.randn((P, H_kv, page, D), generator=g) * 90).clamp(-448, 448).to(F8).view(torch.uint8) for _ in range(2))
    sizes = rng.integers(-7 - spread, -6 + spread, (2, P, H_kv, page // 16)) + (0 if powers else rng.random((2, P, H_kv, page // 16)))
    ks, vs = torch.from_numpy(2.0 ** sizes).float()
    used = torch.zeros((P, page), dtype=torch.bool)
    for b in range(B):
        for r in range(int(kv_len[b]) + (N if nodes is None else int(nodes[b]))):
            used[table[b, r // page], r % page] = True
    for t in (k, v):
        t.permute(0, 2, 1, 3)[~used] = 0x7F
    cells = used.view(P, page // 16, 16).any(2)
    for t in (ks, vs):
        t.permute(0, 2, 1)[~cells] = float("nan")
    q = torch.randn((B, N, H, D), generator=g) * torch.linspace(0.5, 2, H)[None, None, :, None]
    mask = np.stack([datagen.make_random_tree(seed * 100 + b, N, 9)[2] for b in range(B)]) if tree else None
    return dict(q=q.to(dtype), k=k, v=v, ks=ks, vs=vs, table=table, kv_len=kv_len, mask=mask,
                nodes=None if nodes is None else np.asarray(nodes, np.int32), layout=layout)


def values(c, which):
    """What the codes stand for, float64; scales count as they do within their limits."""
    s = torch.nan_to_num(c[which + "s"].double(), nan=2.0 ** -60, posinf=2.0 ** 60).clamp(2.0 ** -60, 2.0 ** 60)
    return c[which].view(F8).double() * s.repeat_interleave(16, 2)[..., None]


def on_gpu(c):
    k, v, q = c["k"].view(F8).cuda(), c["v"].view(F8).cuda(), c["q"].cuda()
    if c["layout"] == "nhd":
        k, v = (t.view(torch.uint8).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3).view(F8) for t in (k, v))
        q = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    return [q, k, v, c["ks"].cuda(), c["vs"].cuda(), to_dev(c["table"]), to_dev(c["kv_len"]),
            None if c["mask"] is None else to_dev(c["mask"].view(np.int32))]


def run(c, window=0, sinks=0, scale=None, want_lse=True):
    args = on_gpu(c)
    B, N, H, D = c["q"].shape
    out = torch.full_like(args[0], 7.0)
    lse = torch.full((B, H, N), 5.0, device="cuda") if want_lse else None
    rest.rest_paged_attention_scaled(*args, 1.0 / math.sqrt(D) if scale is None else scale, window=window, sinks=sinks,
                                     n_nodes=None if c["nodes"] is None else to_dev(c["nodes"]), out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def reference(c, window=0, sinks=0, scale=None):
    D = c["q"].shape[3]
    return plain.attention(c["q"], values(c, "k"), values(c, "v"), c["table"], c["kv_len"], c["mask"],
                           1.0 / math.sqrt(D) if scale is None else scale, window, sinks, c["nodes"])


def near(c, got, got_lse, ref):
    out, lse, A, S = ref
    e = 2.0 ** -8 if c["q"].dtype == BF16 else 2.0 ** -11
    n_keys = int(c["kv_len"].max()) + c["q"].shape[1]
    most = torch.nan_to_num(c["vs"].double(), nan=0.0).clamp(2.0 ** -60, 2.0 ** 60).max()   # as scales count
    rel = (S + 1).transpose(1, 2)[..., None] * 2.0 ** -15
    tol = e * out.abs() + (1 + e) * ((2.0 ** -11 + rel) * A + n_keys * 2.0 ** -31 * 448 * most)
    tol += 2.0 ** -25 if c["q"].dtype == FP16 else 1e-30
    got, live = got.double().cpu(), ~out.isnan()
    over = ((got - out).abs() - tol)[live]
    assert not got[live].isnan().any() and over.max() <= 0, float(over.max())
    if got_lse is not None:
        g, seen = got_lse.double().cpu(), lse.isfinite()
        assert torch.equal(g[lse.isinf()], lse[lse.isinf()])
        if seen.any():
            over = ((g - lse).abs() - (S + 1) * 2.0 ** -16 - lse.abs() * 2.0 ** -22)[seen]
            assert over.max() <= 0, float(over.max())


def check(c, window=0, sinks=0, scale=None):
    out, lse = run(c, window, sinks, scale)
    ref = reference(c, window, sinks, scale)
    near(c, out, lse, ref)
    gone = ref[0].isnan()                          # nodes that do not exist: left as they were
    assert (out.cpu()[gone] == 7.0).all() and (lse.cpu()[ref[1].isnan()] == 5.0).all()
    return out, lse, ref


@pytest.mark.parametrize("B,N,H,H_kv,D,page,L,dtype", [
    (1, 1, 1, 1, 128, 16, 0, BF16),          # one token, nothing before it
    (1, 1, 4, 1, 64, 16, 1, FP16),
    (3, 1, 32, 8, 128, 16, 200, BF16),       # ordinary decoding
    (2, 1, 8, 8, 64, 128, 1000, BF16),
    (1, 1, 8, 1, 128, 32, 2500, FP16),       # one KV head over many SMs
    (2, 1, 16, 1, 128, 64, 333, BF16),       # sixteen heads a KV head, and seventeen
    (2, 1, 17, 1, 64, 64, 333, FP16),
    (2, 3, 5, 1, 128, 16, 500, FP16),        # fifteen rows
    (2, 8, 2, 1, 64, 256, 700, BF16),        # sixteen
    (2, 64, 4, 4, 128, 64, 130, BF16),       # a tree, one KV head per head
    (2, 64, 8, 2, 128, 16, 300, BF16),       # 256 rows a KV head
    (1, 33, 10, 2, 64, 32, 77, FP16),        # five heads a KV head: 165 rows
    (2, 13, 6, 2, 128, 256, 513, BF16),
    (1, 128, 10, 2, 128, 64, 260, BF16),     # 640 rows a KV head
    (1, 256, 3, 1, 64, 16, 100, BF16),       # 768 rows
    (1, 256, 1, 1, 128, 128, 0, FP16),       # only the tree
    (5, 7, 3, 3, 64, 16, 64, BF16),
    (1, 129, 1, 1, 128, 16, 63, FP16),       # one row more than a tile
    (9, 2, 16, 4, 128, 16, 31, FP16),
])
@pytest.mark.parametrize("powers", [True, False])
def test_matches_64_bits(B, N, H, H_kv, D, page, L, dtype, powers):
    check(make(B + N, B, N, H, H_kv, D, page, [L] * B, dtype, powers=powers))


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (1, 0), (5, 70), (3, 1)])
@pytest.mark.parametrize("N,H,H_kv,D,page", [(17, 8, 2, 128, 16), (70, 4, 1, 64, 64), (1, 6, 2, 128, 32), (150, 2, 2, 128, 16),
                                             (4, 3, 1, 128, 64), (2, 16, 2, 64, 16)])
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
                c["k"][c["table"][b, col]] = c["v"][c["table"][b, col]] = 0xFF
                c["ks"][c["table"][b, col]] = c["vs"][c["table"][b, col]] = float("inf")
                c["table"][b, col] = -1 if col % 2 else 12345     # gone, or whatever was left in the entry
    ref = reference(c, window, sinks)
    out, lse = run(c, window, sinks)
    c["vs"] = torch.nan_to_num(c["vs"], posinf=0.0)               # (pages that are gone set no bound)
    near(c, out, lse, ref)


@pytest.mark.parametrize("N,H,D", [(6, 2, 128), (40, 8, 64), (90, 4, 128), (16, 2, 64)])
def test_a_run_of_tokens_without_a_mask(N, H, D):
    for window, sinks in ((0, 0), (16, 2)):
        check(make(N, 2, N, H, 2, D, 32, [100, 3], tree=False), window, sinks)


@pytest.mark.parametrize("N,H,H_kv", [(20, 2, 2), (64, 8, 2), (3, 1, 1), (8, 4, 2)])
def test_rows_that_see_nothing(N, H, H_kv):
    c = make(5, 3, N, H, H_kv, 128, 16, [0, 40, 0])
    c["mask"][:, ::2] = 0
    out, lse, ref = check(c)
    assert (out[0, ::2] == 0).all() and torch.isneginf(lse[0, :, ::2]).all()
    c["mask"][:] = 0                                # a window of one position: a row without its own bit
    check(c, window=1)


@pytest.mark.parametrize("N,H,H_kv,D", [(24, 2, 1, 128), (64, 4, 1, 64), (130, 2, 2, 128), (8, 2, 1, 128), (5, 3, 1, 64)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_what_is_masked_may_be_nan(N, H, H_kv, D, which):
    """NaN in a node's K or V reaches that node and its descendants only; in rows behind the window nobody.
    A NaN in V decides its column whatever the key's probability."""
    c = make(8, 2, N, H, H_kv, D, 16, [150, 90])
    clean = {**c, "k": c["k"].clone(), "v": c["v"].clone()}
    window, sinks = 40, 3
    bad = {0: 2, 1: N // 2}
    for b, node in bad.items():
        for r in [int(c["kv_len"][b]) + node] + list(range(sinks, int(c["kv_len"][b]) - window)):
            p, at = plain.row_of(c["table"], 16, c["k"].shape[0], b, r)
            c[which][p, :, at, 3:9] = 0xFF if r % 2 else 0x7F
            clean[which][p, :, at, 3:9] = 0
    out, lse = run(c, window, sinks)
    ref = reference(clean, window, sinks)
    for b, node in bad.items():
        hit = ((c["mask"][b, :, node >> 5] >> (node & 31)) & 1).astype(bool)
        assert hit.any() and not hit.all()
        got = out[b].float().cpu()
        assert got[hit][..., 3:9].isnan().all() if which == "v" else got[hit].isnan().all()
        if which == "v":
            assert got[hit][..., 9:].isfinite().all() and got[hit][..., :3].isfinite().all()
        for t in (ref[0], ref[2]):
            t[b, torch.from_numpy(hit)] = float("nan")
        ref[1][b, :, torch.from_numpy(hit)] = float("nan")
    near(c, out, lse, ref)


@pytest.mark.parametrize("N,H,H_kv", [(1, 4, 1), (4, 4, 1), (64, 4, 1), (40, 2, 1)])
def test_nan_in_the_prefix_decides_its_column(N, H, H_kv):
    """Seen by all rows, with a probability that rounds to 0."""
    c = make(9, 2, N, H, H_kv, 128, 16, [700, 90])
    p, at = plain.row_of(c["table"], 16, c["k"].shape[0], 0, 333)
    c["v"][p, :, at, 77] = 0x7F
    c["k"][p, :, at] = 0x7E                         # a score far from the others', below or above them
    c["q"] = -c["q"].abs()
    out, lse = run(c)
    assert out[0, ..., 77].isnan().all() and out[0, ..., :77].isfinite().all() and out[0, ..., 78:].isfinite().all()
    assert out[1].isfinite().all() and lse.isfinite().all()


@pytest.mark.parametrize("N,D,H_kv", [(2, 128, 1), (64, 128, 1), (70, 64, 2), (130, 128, 2), (1, 64, 2)])
def test_scores_whose_maximum_keeps_growing(N, D, H_kv):
    c = make(31, 2, N, 2, H_kv, D, 64, [700, 650])
    for b in range(2):
        for r in range(0, int(c["kv_len"][b]) + N, 16):
            p, at = plain.row_of(c["table"], 64, c["k"].shape[0], b, r)
            c["ks"][p, :, at // 16] *= float((1 + 7 * r / 700) * (2.5 if (r // 64) % 5 == 3 else 1))
    check(c)
    check(c, window=150, sinks=70)


@pytest.mark.parametrize("N,H", [(1, 4), (8, 4), (40, 1), (64, 4)])
def test_values_of_very_different_sizes(N, H):
    """Scales of V from 2^-20 to 2^20 from one block to the next, growing or falling."""
    for sign in (1, -1):
        c = make(32, 2, N, H, 1, 128, 32, [400, 77])
        for b in range(2):
            for i, r in enumerate(range(0, int(c["kv_len"][b]) + N, 16)):
                p, at = plain.row_of(c["table"], 32, c["k"].shape[0], b, r)
                c["vs"][p, :, at // 16] = 2.0 ** (sign * (i * 40 // 26 - 20))
        check(c)


@pytest.mark.parametrize("N,H", [(1, 4), (16, 1), (30, 4)])
@pytest.mark.parametrize("odd", [0.0, -3.0, float("nan"), 2.0 ** -80, 1e-38])
def test_scales_that_are_none(odd, N, H):
    """They count as the nearest limit: such a block's keys score 0, its values vanish, and its probabilities count."""
    c = make(33, 1, N, H, 1, 64, 16, [200])
    p, _ = plain.row_of(c["table"], 16, c["k"].shape[0], 0, 48)
    c["ks"][p], c["vs"][p] = odd, odd
    check(c)
    c = make(34, 1, N, H, 1, 64, 16, [5])           # nothing but such blocks
    c["ks"][:], c["vs"][:] = odd, odd
    out, lse, ref = check(c)
    assert (out.float().abs() < 2.0 ** -24).all()


def test_pools_beyond_32_bit_offsets():
    for B, N, H, H_kv in ((2, 4, 8, 8), (2, 40, 8, 8)):
        D, page = 128, 128
        P = (1 << 32) // (H_kv * page * D) + 40
        c = make(12, B, N, H, H_kv, D, page, [300, 500])
        far = {int(p): P - 1 - i for i, p in enumerate(sorted(set(c["table"].ravel().tolist())))}
        k, v = (torch.zeros((P, H_kv, page, D), dtype=torch.uint8, device="cuda") for _ in range(2))
        ks, vs = (torch.ones((P, H_kv, page // 16), device="cuda") for _ in range(2))
        for p, z in far.items():
            k[z], v[z], ks[z], vs[z] = c["k"][p].cuda(), c["v"][p].cuda(), c["ks"][p].cuda(), c["vs"][p].cuda()
        assert min(far.values()) * H_kv * page * D > 1 << 32
        table = np.vectorize(far.get)(c["table"]).astype(np.int32)
        out = rest.rest_paged_attention_scaled(c["q"].cuda(), k.view(F8), v.view(F8), ks, vs, to_dev(table), to_dev(c["kv_len"]),
                                               to_dev(c["mask"].view(np.int32)), 1 / math.sqrt(D))
        near(c, out, None, reference(c))


@pytest.mark.parametrize("N", [1, 20])
def test_other_streams_captures_and_shared_scratch(N):
    """Calls on a side stream, and a captured step replayed on new inputs while an eager call of
    another shape runs in between with its own scratch: the same bits as plain calls."""
    a, b = make(1, 2, N, 4, 1, 128, 16, [400, 90]), make(2, 1, 3, 2, 2, 128, 16, [900])
    want_a, want_b = run(a), run(b)
    args = on_gpu(a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rest.rest_paged_attention_scaled(*args, 1 / math.sqrt(128), stream=side)
    side.synchronize()
    assert torch.equal(got, want_a[0])
    out, lse = torch.zeros_like(args[0]), torch.zeros((2, 4, N), device="cuda")
    ws = torch.full((max(rest.paged_attention_workspace_bytes(2, 4, 1, N, 128), 16),), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rest.rest_paged_attention_scaled(*args, 1 / math.sqrt(128), out=out, lse=lse, workspace=ws)
    keep = args[0].clone()
    for _ in range(3):
        args[0].copy_(keep * 0.5)
        graph.replay()
        assert torch.equal(run(b)[0], want_b[0])
        args[0].copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_a[0]) and torch.equal(lse, want_a[1])


def test_many_short_contexts():
    lens = np.random.default_rng(2).integers(0, 40, 700)
    check(make(44, 700, 1, 2, 1, 64, 16, lens, FP16))
    check(make(45, 300, 3, 2, 2, 128, 16, lens[:300]), window=8, sinks=2)
    check(make(46, 200, 20, 2, 2, 128, 16, lens[:200]), window=8, sinks=2)


@pytest.mark.parametrize("N,H,D", [(1, 8, 128), (64, 8, 64), (100, 8, 128), (9, 8, 128)])
def test_agrees_with_the_16_bit_call_on_the_same_values(N, H, D):
    """Values that bf16 holds exactly: both calls are within their bounds of the same exact result."""
    c = make(77, 2, N, H, 4, D, 64, [500, 123], powers=True)
    for t in (c["k"], c["v"]):
        t[t == 0x7F] = 0
    c["ks"], c["vs"] = (torch.nan_to_num(t, nan=1.0) for t in (c["ks"], c["vs"]))
    out, _ = run(c)
    args = on_gpu(c)
    k, v = (values(c, w).to(BF16).cuda() for w in "kv")
    other = rest.rest_paged_attention(args[0], k, v, *args[5:], 1 / math.sqrt(D))
    ref = reference(c)
    near(c, out, None, ref)
    plain.assert_attention(other, None, ref, BF16, 600)


@pytest.mark.parametrize("N,D,window", [(66, 128, 0), (66, 128, 150), (66, 64, 0), (40, 128, 0), (4, 128, 0), (1, 128, 0), (20, 64, 0)])
def test_values_that_arrive_late(N, D, window):
    """Keys in the cache, values not: the last two products of a piece are both under way at its end."""
    B, H, H_kv, page = 30, 8, 4, 64
    nodes = [N if b % 3 else max(N // 2, 1) for b in range(B)]
    c = make(N + D, B, N, H, H_kv, D, page, [150 + 37 * (b % 7) for b in range(B)], BF16, nodes)
    c["q"] = (c["q"].float() * 2).to(BF16)         # peaked rows: a tile that is left out shows
    ref = reference(c, window)
    args = on_gpu(c)
    n = to_dev(c["nodes"])
    flush = torch.empty(256 << 20, dtype=torch.int8, device="cuda")
    for _ in range(6):
        out = torch.full_like(args[0], 7.0)
        lse = torch.full((B, H, N), 5.0, device="cuda")
        flush.zero_()
        args[1].view(torch.int16).sum()
        rest.rest_paged_attention_scaled(*args, 1 / math.sqrt(D), window=window, n_nodes=n, out=out, lse=lse)
        near(c, out, lse, ref)


@pytest.mark.parametrize("N,G,D", [(128, 5, 128), (128, 5, 64), (150, 2, 128), (200, 4, 128)])
def test_row_blocks_with_shares_of_their_own(N, G, D):
    """Several row blocks, the last one lower; contexts whose nodes leave it, or all but the first one, empty."""
    lens = [700, 0, 65, 1300, 333, 4, 64, 900]
    nodes = [N, 1, N // 2, N - 1, 0, N, 64 // G, N // 3]
    check(make(N + G, len(lens), N, 2 * G, 2, D, 32, lens, BF16, nodes))
    check(make(N - G, 1, N, 2 * G, 2, D, 32, lens[:1], BF16), 100, 3)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
@pytest.mark.parametrize("N,G,H_kv,D,B", [(64, 4, 2, 128, 40), (140, 1, 3, 64, 40), (33, 4, 8, 128, 9), (64, 4, 1, 128, 3),
                                          (4, 4, 2, 128, 40), (16, 1, 3, 64, 20)])
def test_contexts_with_few_and_many_rows(N, G, H_kv, D, B, window, sinks):
    rng = np.random.default_rng(N + B)
    nodes = [int(rng.choice([0, 1, N // 3, N // 2, N - 1, N])) for _ in range(B)]
    lens = [int(rng.choice([0, 1, 64, 63, 200, 391])) for _ in range(B)]
    check(make(N + B, B, N, G * H_kv, H_kv, D, 16, lens, BF16, nodes), window, sinks)


@pytest.mark.parametrize("length", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 4097])
@pytest.mark.parametrize("N,H,H_kv", [(1, 4, 2), (6, 2, 1), (30, 2, 2)])
def test_every_key_counts_once(length, N, H, H_kv):
    """Equal scores and values of 1: the output is 1, the sum the number of keys."""
    c = make(50, 2, N, H, H_kv, 128, 16, [length, length // 2], tree=False)
    c["k"][:], c["v"][:], c["vs"][:] = 0, 0x38, 1.0
    c["v"][..., 1::2] = 0xB8
    out, lse = run(c)
    assert (out[..., ::2] == 1).all() and (out[..., 1::2] == -1).all()
    n = torch.tensor(c["kv_len"])[:, None, None] + 1 + torch.arange(N)[None, None]
    assert (lse.cpu().double() - n.double().log()).abs().max() <= 2.0 ** -16


def refuse(**kw):
    c = make(60, 2, 3, 4, 2, 64, 16, [30, 5])
    args = on_gpu(c)
    for name, i in (("q", 0), ("k", 1), ("v", 2), ("ks", 3), ("vs", 4), ("table", 5), ("kv_len", 6), ("mask", 7)):
        if name in kw:
            args[i] = kw.pop(name)(args[i])
    with pytest.raises(rest.RestError):
        rest.rest_paged_attention_scaled(*args, 0.125, **kw)


def test_refusals():
    refuse(q=lambda t: t.float())
    refuse(k=lambda t: t.view(torch.uint8))
    refuse(v=lambda t: t[:-1])
    refuse(ks=lambda t: t.double())
    refuse(vs=lambda t: t[:, :, :0])
    refuse(ks=lambda t: t.cpu())
    refuse(ks=lambda t: t.transpose(0, 1).contiguous().transpose(0, 1))
    refuse(kv_len=lambda t: t.long())
    refuse(mask=lambda t: t.float())
    refuse(window=-1)
    refuse(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    refuse(lse=torch.zeros((2, 4, 2), device="cuda"))
