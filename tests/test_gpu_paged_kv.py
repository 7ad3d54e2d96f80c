"""Rows and pages of a paged cache against a plain model: every result is an integer or a moved
16-bit value, so all comparisons are exact."""
import numpy as np
import pytest
import torch

import paged_util as plain
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


def pool(rng, P, H_kv, page, D, layout="hnd", dtype=torch.bfloat16):
    """A pool tensor [P,H_kv,page,D] and its bits as numpy; "nhd": rows before heads in memory;
    "gap": K and V interleaved in one allocation."""
    raw = rng.integers(0, 1 << 15, (2, P, H_kv, page, D)).astype(np.int16)
    t = torch.from_numpy(raw).to("cuda:0")
    if layout == "nhd":
        t = t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    elif layout == "gap":
        t = t.transpose(0, 1).contiguous().transpose(0, 1)
    return t[0].view(dtype), t[1].view(dtype), raw[0].copy(), raw[1].copy()


def same(t, raw):
    return np.array_equal(t.view(torch.int16).cpu().numpy(), raw)


def tables(rng, B, W, P, holes=()):
    t = rng.permutation(P)[:B * W].reshape(B, W).astype(np.int32)
    for b, c, value in holes:
        t[b, c] = value
    return t


@pytest.mark.parametrize("B,N,H_kv,page,D,layout", [
    (1, 1, 1, 16, 64, "hnd"), (3, 7, 5, 16, 128, "nhd"), (2, 64, 32, 64, 128, "hnd"), (5, 33, 3, 32, 64, "gap"),
    (2, 256, 1, 256, 128, "hnd"), (4, 2, 65, 128, 64, "nhd"),
])
def test_rows_are_written_and_committed(B, N, H_kv, page, D, layout):
    rng = np.random.default_rng(B * 100 + N)
    W = -(-(3 * page + N) // page) + 1
    P = B * W + 3
    k, v, k0, v0 = pool(rng, P, H_kv, page, D, layout, torch.float16 if D == 64 else torch.bfloat16)
    table = tables(rng, B, W, P, holes=[(0, 1, -1), (B - 1, W - 2, P)])      # pages that do not exist
    kv_len = rng.integers(0, 3 * page + 1, B).astype(np.int32)
    nodes = rng.integers(0, N + 1, B).astype(np.int32)
    new = rng.integers(0, 1 << 15, (2, B, N, H_kv, D)).astype(np.int16)
    k_new, v_new = (torch.from_numpy(x).to("cuda:0").view(k.dtype) for x in new)
    for n in (nodes, None):
        rest.rest_paged_kv_write(k, v, to_dev(table), to_dev(kv_len), k_new, v_new,
                                 n_nodes=None if n is None else to_dev(n))
        plain.write(k0, table, kv_len, new[0], n), plain.write(v0, table, kv_len, new[1], n)
        assert same(k, k0) and same(v, v0)
    depth = min(N, 16)
    path = np.full((B, depth), -1, np.int32)
    lens = rng.integers(0, depth + 1, B).astype(np.int32)
    for b in range(B):
        path[b, :lens[b]] = np.sort(rng.permutation(N)[:lens[b]])
    lens[0] = depth
    path[0] = np.sort(rng.permutation(N)[:depth])
    d_len = to_dev(kv_len)
    rest.rest_paged_kv_commit(k, v, to_dev(table), d_len, to_dev(path), to_dev(lens), N, new_kv_len=d_len)
    plain.commit(k0, table, kv_len, path, lens, N), plain.commit(v0, table, kv_len, path, lens, N)
    assert same(k, k0) and same(v, v0)
    assert np.array_equal(d_len.cpu().numpy(), kv_len + lens)


def test_strided_rows_and_tables():
    rng = np.random.default_rng(9)
    k, v, k0, v0 = pool(rng, 9, 4, 16, 128)
    wide = np.full((2, 11), 99, np.int32)
    wide[:, :4] = tables(rng, 2, 4, 9)
    table = to_dev(wide)[:, :4]
    new = torch.from_numpy(rng.integers(0, 1 << 15, (2, 4, 2, 2, 5, 128)).astype(np.int16)).to("cuda:0")
    k_new, v_new = (new[i].permute(1, 2, 0, 3, 4)[:, :, :, 2].view(k.dtype) for i in (0, 1))    # [B,N,H_kv,D]
    kv_len = np.array([15, 30], np.int32)
    rest.rest_paged_kv_write(k, v, table, to_dev(kv_len), k_new, v_new)
    for raw, x in ((k0, k_new), (v0, v_new)):
        plain.write(raw, wide[:, :4], kv_len, x.contiguous().view(torch.int16).cpu().numpy())
    assert same(k, k0) and same(v, v0)


@pytest.mark.parametrize("H_kv,page,D,layout", [(1, 16, 64, "hnd"), (8, 16, 128, "nhd"), (3, 128, 64, "gap"),
                                                (5, 256, 128, "hnd")])
def test_pages_are_copied(H_kv, page, D, layout):
    rng = np.random.default_rng(page + H_kv)
    k, v, k0, v0 = pool(rng, 12, H_kv, page, D, layout)
    src = np.array([3, -1, 5, 3, 12, 7], np.int32)
    dst = np.array([0, 1, 2, 11, 4, -1], np.int32)
    rest.rest_pages_copy(k, v, to_dev(src), to_dev(dst))
    for raw in (k0, v0):
        for a, z in ((3, 0), (5, 2), (3, 11)):
            raw[z] = raw[a]
    assert same(k, k0) and same(v, v0)


def pages_state(rng, B, W, P, page, used):
    """Contexts 0..used-1 hold random lengths, the others nothing."""
    table = np.full((B, W), -1, np.int32)
    n_pages, kv_len, refs = np.zeros(B, np.int32), np.zeros(B, np.int32), np.zeros(P, np.int32)
    order = rng.permutation(P)
    at = 0
    for b in range(used):
        kv_len[b] = rng.integers(0, (W - 1) * page)
        n = -(-int(kv_len[b]) // page)
        n_pages[b] = n
        table[b, :n] = order[at:at + n]
        refs[order[at:at + n]] = 1
        at += n
    return refs, table, n_pages, kv_len


def check(dev, host):
    for t, a in zip(dev, host):
        assert np.array_equal(t.cpu().numpy(), a)


@pytest.mark.parametrize("B,used,W,P,page,F", [(6, 2, 5, 40, 16, 4), (40, 9, 7, 64, 32, 30), (1100, 70, 9, 1500, 64, 1024),
                                               (12, 1, 3, 3, 16, 9), (300, 20, 40, 5000, 256, 200)])
def test_fork_reserve_release(B, used, W, P, page, F):
    rng = np.random.default_rng(B + F)
    refs, table, n_pages, kv_len = pages_state(rng, B, W, max(P, used * W), page, used)
    if F == 9:
        kv_len[0], n_pages[0], table[0, 0], refs[:] = page // 2, 1, 1, [0, 1, 0]   # room for two of nine forks
    P = len(refs)
    dev = [to_dev(x) for x in (refs, table, n_pages, kv_len)]
    parents = rng.integers(-1, used + 2, F).astype(np.int32)
    if F == 9:
        parents[:] = 0
    children = (used + np.arange(F) % (B - used)).astype(np.int32)            # some named twice
    children[F // 2] = B + 1 if F != 9 else children[F // 2]
    got = rest.rest_pages_fork(*dev, to_dev(parents), to_dev(children), page)
    want = plain.fork(refs, table, n_pages, kv_len, parents, children, page)
    check(got, want), check(dev, (refs, table, n_pages, kv_len))
    assert (want[2] == 0).any() and (F != 9 or (want[2] == 4).any())

    need = (kv_len + rng.integers(-2, 2 * page, B)).astype(np.int32)
    need[0] = W * page + 1                                                    # more than its table holds
    st = rest.rest_pages_reserve(dev[0], dev[1], dev[2], to_dev(need), page)
    assert np.array_equal(st.cpu().numpy(), plain.reserve(refs, table, n_pages, need, page))
    check(dev, (refs, table, n_pages, kv_len))

    for window, sinks in ((2 * page, 4), (0, 0), (1, 0)):
        keep = np.maximum(kv_len - rng.integers(0, page, B), 0).astype(np.int32)
        keep[1::7] = -1
        rest.rest_pages_release(dev[0], dev[1], dev[2], to_dev(keep), page, window=window, sinks=sinks)
        plain.release(refs, table, n_pages, keep, page, window, sinks)
        check(dev, (refs, table, n_pages, kv_len))
    everything = np.zeros(B, np.int32)
    rest.rest_pages_release(dev[0], dev[1], dev[2], to_dev(everything), page)
    plain.release(refs, table, n_pages, everything, page)
    check(dev, (refs, table, n_pages, kv_len))
    assert refs.sum() == 0 and n_pages.sum() == 0


def test_reserve_runs_out_of_pages_and_gives_all_or_nothing():
    page, W, P, B = 16, 6, 11, 5
    refs, table = np.zeros(P, np.int32), np.full((B, W), -1, np.int32)
    refs[[0, 3, 4]] = 2
    n_pages = np.zeros(B, np.int32)
    need = np.array([3 * page, 2 * page + 1, 4 * page, 0, 1], np.int32)       # 3 + 3 of 8, then 4 too many
    dev = [to_dev(x) for x in (refs, table, n_pages)]
    st = rest.rest_pages_reserve(*dev, to_dev(need), page)
    assert st.tolist() == [0, 0, 4, 0, 4]
    assert np.array_equal(plain.reserve(refs, table, n_pages, need, page), st.cpu().numpy())
    check(dev, (refs, table, n_pages))
    assert table[0, :3].tolist() == [1, 2, 5] and table[1, :3].tolist() == [6, 7, 8]


def test_a_captured_step_replays():
    """Reserve, write, commit and release captured once and replayed on changed inputs."""
    rng = np.random.default_rng(4)
    B, N, page, W, P = 3, 5, 16, 4, 20
    k, v, k0, v0 = pool(rng, P, 2, page, 64)
    refs, table, n_pages, kv_len = pages_state(rng, B, W, P, page, B)
    kv_len[:] = kv_len // 2
    dev = [to_dev(x) for x in (refs, table, n_pages, kv_len)]
    new = to_dev(rng.integers(0, 1 << 15, (2, B, N, 2, 64)).astype(np.int16))
    nodes, lens = to_dev(np.tile(np.array([0, 2], np.int32), (B, 1))), to_dev(np.array([2, 0, 1], np.int32))
    need, st = torch.empty_like(dev[3]), torch.empty_like(dev[3])

    def step(stream=None):
        torch.add(dev[3], N, out=need)
        rest.rest_pages_reserve(dev[0], dev[1], dev[2], need, page, status=st, stream=stream)
        rest.rest_paged_kv_write(k, v, dev[1], dev[3], new[0].view(k.dtype), new[1].view(k.dtype), stream=stream)
        rest.rest_paged_kv_commit(k, v, dev[1], dev[3], nodes, lens, N, new_kv_len=dev[3], stream=stream)
        rest.rest_pages_release(dev[0], dev[1], dev[2], dev[3], page, stream=stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        new.copy_(to_dev(rng.integers(0, 1 << 15, tuple(new.shape)).astype(np.int16)))
        fresh = new.cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        plain.reserve(refs, table, n_pages, kv_len + N, page)
        for raw, x in ((k0, fresh[0]), (v0, fresh[1])):
            plain.write(raw, table, kv_len, x)
            plain.commit(raw, table, kv_len, nodes.cpu().numpy(), lens.cpu().numpy(), N)
        kv_len += lens.cpu().numpy()
        plain.release(refs, table, n_pages, kv_len, page)
        check(dev, (refs, table, n_pages, kv_len))
        assert same(k, k0) and same(v, v0)
