"""rest_paged_kv_append and _append_scaled, rest_paged_kv_commit_scaled and rest_pages_copy_scaled against plain models.
Codes and scales have to be equal: both sides round values that differ by a few 2^-53."""
import numpy as np
import pytest
import torch

import datagen
import paged_util
import paper_2311_08252_b200 as rest
import scaled_util as plain

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def step(seed, B, N, H, H_kv, D, F, dtype, kv_len, page, spread=3):
    """A step's rows, some louder than others, and the positions of a random tree."""
    rng = np.random.default_rng(seed)
    loud = 2.0 ** rng.integers(-spread, spread + 1, (B, N, 1, 1))
    k, v = (torch.from_numpy(rng.normal(size=(B, N, H_kv, D)) * loud).to(dtype) for _ in range(2))
    q = torch.from_numpy(rng.normal(size=(B, N, H, D))).to(dtype)
    pos = np.asarray(kv_len)[:, None] + rng.integers(0, 9, (B, N))
    freq = (10000.0 ** (-np.arange(F) / max(F, 1))).astype(np.float32)
    return rng, q, k, v, pos.astype(np.int32), freq


CASES = [  # B, N, H, H_kv, D, F, dtype, kv_len, page, nodes, interleaved, layout
    (1, 1, 4, 1, 128, 64, BF16, [2048], 16, None, False, "hnd"),
    (4, 1, 8, 2, 64, 32, FP16, [0, 15, 16, 700], 32, None, True, "nhd"),
    (3, 64, 8, 8, 128, 64, BF16, [5, 16, 127], 64, [64, 1, 33], False, "gap"),
    (2, 33, 5, 1, 128, 32, FP16, [0, 31], 128, [0, 33], True, "hnd"),
    (2, 20, 6, 2, 64, 13, BF16, [250, 7], 256, [19, 20], False, "nhd"),
    (1, 256, 3, 3, 64, 32, BF16, [9], 16, None, False, "hnd"),
    (40, 17, 2, 2, 128, 64, FP16, list(range(40)), 16, None, True, "hnd"),
    (2, 16, 0, 4, 128, 0, BF16, [3, 48], 16, None, False, "hnd"),
    (300, 17, 3, 1, 64, 32, BF16, [7 * b % 50 for b in range(300)], 32, [b % 18 for b in range(300)], False, "hnd"),
]


def live(c):
    return np.full(c[0], c[1]) if c[9] is None else np.asarray(c[9])


@pytest.mark.parametrize("c", CASES)
def test_16_bit_pages(c):
    B, N, H, H_kv, D, F, dtype, kv_len, page, nodes, inter, layout = c
    rng, q, k, v, pos, freq = step(B + N, *c[:9])
    W = -(-(max(kv_len) + N) // page)
    P = B * W + 1
    raw = rng.integers(0, 1 << 14, (2, P, H_kv, page, D)).astype(np.int16)
    t = torch.from_numpy(raw).cuda()
    if layout == "nhd":
        t = t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    pk, pv = t[0].view(dtype), t[1].view(dtype)
    table = plain.tables(rng, B, W, P)
    table[0, 0] = -1                                    # the first context's first rows have no page
    turn = dict(positions=cuda(pos), inv_freq=cuda(freq), interleaved=inter, amplitude=1.5) if F else {}
    nn = None if nodes is None else cuda(np.asarray(nodes, np.int32))
    qd = q.cuda() if H else None
    q_out = torch.full_like(qd, 7) if H else None
    got = rest.rest_paged_kv_append(pk, pv, cuda(table), cuda(np.asarray(kv_len, np.int32)), k.cuda(), v.cuda(), n_nodes=nn,
                                    q=qd, q_out=q_out, **turn)
    rotated = rest.rest_rotary(k.cuda(), **turn) if F else k.cuda()
    for pool, want, new in ((pk, raw[0], rotated), (pv, raw[1], v)):
        paged_util.write(want, table, kv_len, new.view(torch.int16).cpu().numpy(), nodes)
        assert np.array_equal(pool.view(torch.int16).cpu().numpy(), want)
    if H:
        want = rest.rest_rotary(qd, **turn)
        for b, n in enumerate(live(c)):
            assert torch.equal(got[b, :n], want[b, :n]) and (got[b, n:] == 7).all()


@pytest.mark.parametrize("c", CASES)
def test_scaled_pages(c):
    B, N, H, H_kv, D, F, dtype, kv_len, page, nodes, inter, layout = c
    rng, q, k, v, pos, freq = step(B * N, *c[:9])
    W = -(-(max(kv_len) + N) // page)
    P = B * W + 1
    pk, pv, ks, vs, raw, scales = plain.pool(rng, P, H_kv, page, D, layout)
    table = plain.tables(rng, B, W, P)
    table[B - 1, W - 1] = P + 3                         # no such page
    turn = dict(positions=cuda(pos), inv_freq=cuda(freq), interleaved=inter, amplitude=0.75) if F else {}
    qd = q.cuda() if H else None
    got = rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), cuda(np.asarray(kv_len, np.int32)), k.cuda(),
                                           v.cuda(), n_nodes=None if nodes is None else cuda(np.asarray(nodes, np.int32)),
                                           q=qd, q_out=qd, **turn)
    kk = k.double().numpy()
    kk = plain.turn(kk, pos, freq, inter, 0.75) if F else kk
    for i, (codes, sc, new) in enumerate(((pk, ks, kk), (pv, vs, v.double().numpy()))):
        plain.write(raw[i], scales[i], table, kv_len, new, live(c))
        assert np.array_equal(sc.cpu().numpy(), scales[i])
        assert plain.same_codes(codes, raw[i])
    if H:                                               # in place: rows behind the tree as they were
        want = rest.rest_rotary(q.cuda(), **turn)
        for b, n in enumerate(live(c)):
            assert got is qd and torch.equal(qd[b, :n], want[b, :n]) and torch.equal(qd[b, n:].cpu(), q[b, n:])


def scaled_state(seed, B, H_kv, D, page, kv_len, N):
    rng = np.random.default_rng(seed)
    W = -(-(max(kv_len) + N) // page)
    P = B * W + 2
    return (rng, *plain.pool(rng, P, H_kv, page, D), plain.tables(rng, B, W, P))


@pytest.mark.parametrize("value", [0.0, 1e-30, 448.0, 448.0000001, 449.0, 3e38, float("nan"), float("inf"), -float("inf")])
def test_values_at_the_ends(value):
    """One value among zeros: zero and tiny ones take the least scale, 448 times a power of two the power itself, huge
    ones saturate, what is not finite becomes NaN and has no part in the scale."""
    kv_len = [20]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(1, 1, 2, 64, 16, kv_len, 3)
    new = torch.zeros((1, 3, 2, 64), dtype=BF16)
    new[0, 1, 0, 5] = value
    new[0, 2, 1, 9] = 2.0
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), cuda(np.array(kv_len, np.int32)), new.cuda(), new.cuda())
    for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
        plain.write(raw[i], scales[i], table, kv_len, new.double().numpy(), [3])
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 0.3, 2.0 ** -70, 2.0 ** 70])
def test_older_rows_under_other_scales(scale):
    """A scale that no power of two or no scale at all: counts as documented, older rows are requantised by it."""
    kv_len = [5, 16]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(2, 2, 1, 128, 16, kv_len, 2)
    ks.fill_(scale)
    vs.fill_(scale)
    scales[:] = scale
    new = torch.from_numpy(rng.normal(size=(2, 2, 1, 128))).to(BF16)
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), cuda(np.array(kv_len, np.int32)), new.cuda(), new.cuda())
    for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
        plain.write(raw[i], scales[i], table, kv_len, new.double().numpy(), [2, 2])
        assert np.array_equal(sc.cpu().numpy(), np.float32(scales[i]), equal_nan=True)
        g, w = plain.decode(codes.view(torch.uint8).cpu().numpy()), plain.decode(raw[i])
        if scale == 0.3:   # quotients and products by 0.3 are rounded to 32 bits before they are to codes: a border may be crossed
            assert (g != w).mean() < 1e-3 and np.abs(g - w).max() <= 32
        else:
            assert np.array_equal(g, w, equal_nan=True)


@pytest.mark.parametrize("B,N,H_kv,D,page,depth,lens", [
    (1, 64, 8, 128, 16, 10, [2048]), (5, 33, 2, 64, 32, 16, [0, 1, 15, 16, 100]), (130, 9, 1, 128, 64, 5, None),
    (3, 256, 32, 64, 256, 16, [300, 7, 64]), (2, 1, 3, 128, 128, 1, [31, 32])])
@pytest.mark.parametrize("alias", [False, True])
def test_commit(B, N, H_kv, D, page, depth, lens, alias):
    lens = list(range(B)) if lens is None else lens
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(B * N, B, H_kv, D, page, lens, N)
    nodes = np.stack([np.sort(rng.choice(np.arange(max(N, depth)), depth, replace=False)) for _ in range(B)]).astype(np.int32)
    n = rng.integers(0, depth + 1, B).astype(np.int32)
    n[0] = depth
    kv = cuda(np.array(lens, np.int32))
    out = kv if alias else torch.zeros_like(kv)
    rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, cuda(table), kv, cuda(nodes), cuda(n), N, new_kv_len=out)
    for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
        plain.commit(raw[i], scales[i], table, lens, nodes, n, N)
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])
    assert out.cpu().tolist() == [a + int(b) for a, b in zip(lens, n)]


def test_commit_keeps_to_its_limits():
    """Lengths and nodes out of range are clamped, contexts without pages or with negative lengths stay as they are."""
    lens = [3, -1, 40, 20]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(11, 4, 2, 64, 16, lens, 8)
    table[2] = -1
    nodes = np.array([[-3, 99, 2], [0, 1, 2], [0, 1, 2], [5, 6, 7]], np.int32)
    n = np.array([3, 3, 3, 99], np.int32)
    rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, cuda(table), cuda(np.array(lens, np.int32)), cuda(nodes), cuda(n), 8)
    for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
        plain.commit(raw[i], scales[i], table, lens, nodes, n, 8)
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])


@pytest.mark.parametrize("P,H_kv,page,D,layout", [(9, 8, 16, 128, "hnd"), (6, 3, 256, 64, "nhd"), (40, 1, 32, 64, "gap")])
def test_copy(P, H_kv, page, D, layout):
    rng = np.random.default_rng(P)
    pk, pv, ks, vs, raw, scales = plain.pool(rng, P, H_kv, page, D, layout)
    src, dst = np.array([0, 3, -1, 2, P, 1], np.int32), np.array([4, 1, 2, P, 3, 1], np.int32)
    dst[5] = 1
    src[1], dst[1] = 3, P - 1
    rest.rest_pages_copy_scaled(pk, pv, ks, vs, cuda(src), cuda(dst))
    for a, z in zip(src, dst):
        if 0 <= a < P and 0 <= z < P:
            raw[:, z], scales[:, z] = raw[:, a], scales[:, a]
    for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])


def test_append_then_commit_is_append_of_the_path():
    """The accepted rows of an appended draft, committed, are what appending the path alone gives where no branch
    that was refused is louder than it (all scales are the same then)."""
    kv_len = [37, 16]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(21, 2, 2, 64, 32, kv_len, 24)
    k2, v2, ks2, vs2 = pk.clone(), pv.clone(), ks.clone(), vs.clone()
    parents = datagen.make_random_tree(5, 24, 9)[0]
    path = [23]
    while parents[path[0]] >= 0:
        path.insert(0, int(parents[path[0]]))
    new = torch.from_numpy(rng.uniform(1, 1.7, (2, 24, 2, 64))).to(BF16).cuda()
    kv, nodes = cuda(np.array(kv_len, np.int32)), cuda(np.array([path] * 2, np.int32))
    lens = cuda(np.full(2, len(path), np.int32))
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), kv, new, new)
    rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, cuda(table), kv, nodes, lens, 24)
    alone = new[:, path].contiguous()
    rest.rest_paged_kv_append_scaled(k2, v2, ks2, vs2, cuda(table), kv, alone, alone)
    for b, L in enumerate(kv_len):
        for r in range(L // 16 * 16, L + len(path)):
            p, at = paged_util.row_of(table, 32, pk.shape[0], b, r)
            for x, y, s, t in ((pk, k2, ks, ks2), (pv, v2, vs, vs2)):
                assert torch.equal(s[p, :, at // 16], t[p, :, at // 16])
                assert torch.equal(x[p, :, at].view(torch.uint8), y[p, :, at].view(torch.uint8))
