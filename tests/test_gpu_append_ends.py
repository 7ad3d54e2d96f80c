"""The appends and the commit in codes where values, pages and refused drafts are at their ends, against the plain models."""
import numpy as np
import pytest
import torch

import paged_util
import paper_2311_08252_b200 as rest
import scaled_util as plain
from test_gpu_append import BF16, cuda, scaled_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F,amplitude,value", [(32, 1.0, 3.3e38), (32, 2.0, 2e38), (13, 1.0, 3.3e38), (13, -3.0, 3e38), (32, 1e6, 1e37)])
def test_finite_values_that_32_bits_do_not_hold(F, amplitude, value, interleaved):
    """Pairs that a rotation or the amplitude takes beyond the largest 32-bit number saturate as other large ones do;
    what is not finite beside them becomes NaN."""
    kv_len = [20]
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(5, 1, 2, 64, 16, kv_len, 4)
    new = torch.zeros((1, 4, 2, 64), dtype=BF16)
    one, two = (6, 7) if interleaved else (3, F + 3)
    new[0, 1, 0, one], new[0, 1, 0, two] = value, value
    new[0, 2, 1, one], new[0, 2, 1, two] = -value, value
    new[0, 3, 1, one + 2 if interleaved else one + 1] = float("inf")
    pos = np.array([[0, 1, 2, 3]], np.int32)
    freq = np.full(F, 0.7853981633974483, np.float32)
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), cuda(np.array(kv_len, np.int32)), new.cuda(), new.cuda(),
                                     cuda(pos), cuda(freq), interleaved, amplitude)
    with np.errstate(invalid="ignore"):
        k = plain.turn(new.double().numpy(), pos, freq, interleaved, amplitude)
    assert np.abs(k[np.isfinite(k)]).max() > np.finfo(np.float32).max
    for i, (codes, sc, x) in enumerate(((pk, ks, k), (pv, vs, new.double().numpy()))):
        plain.write(raw[i], scales[i], table, kv_len, x, [4])
        assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("F", [5, 8, 13, 32])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_is_not_finite_stays_with_its_pair(F, interleaved, scaled, bad):
    """In either half of a pair, at the border of the halves, in lanes that hold turned and copied elements."""
    pairs = sorted({0, F // 2, F - 1})
    for f in pairs:
        for second in (0, 1):
            kv_len = [18]
            rng, pk, pv, ks, vs, raw, scales, table = scaled_state(6, 1, 2, 64, 16, kv_len, 3)
            if not scaled:
                pk, pv = (torch.zeros(pk.shape, dtype=BF16, device="cuda") for _ in range(2))
            new = torch.from_numpy(rng.normal(size=(1, 3, 2, 64))).to(BF16)
            where = [2 * f, 2 * f + 1] if interleaved else [f, F + f]
            new[0, 1, 1, where[second]] = bad
            turn = (cuda(np.array([[3, 4, 5]], np.int32)), cuda(np.full(F, 0.7, np.float32)), interleaved)
            args = (cuda(table), cuda(np.array(kv_len, np.int32)), new.cuda(), torch.zeros_like(new).cuda(), *turn)
            if scaled:
                rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, *args)
            else:
                rest.rest_paged_kv_append(pk, pv, *args)
            for r in range(3):
                p, at = paged_util.row_of(table, 16, pk.shape[0], 0, 18 + r)
                odd = (~pk[p, :, at].float().isfinite()).nonzero().tolist()
                assert odd == ([[1, w] for w in where] if r == 1 else [])
            assert pv.float().isfinite().all()


def plain_commit(codes, scales, table, kv_len, nodes, lens, N):
    """Path rows whose source or target page does not exist are left alone and have no part in a scale."""
    P, H, page, D = codes.shape
    old, old_scales = codes.copy(), scales.copy()
    for b in range(len(kv_len)):
        L = int(kv_len[b])
        n = min(max(int(lens[b]), 0), nodes.shape[1])
        source = [paged_util.row_of(table, page, P, b, L + min(max(int(nodes[b, i]), 0), N - 1)) for i in range(n)]
        for first in range(L // 16 * 16, L + n, 16):
            at = paged_util.row_of(table, page, P, b, first)
            rows = [i for i in range(max(first - L, 0), min(first + 16 - L, n)) if source[i]]
            if at is None or not rows:
                continue
            p, r = at
            for h in range(H):
                v = np.stack([plain.decode(old[source[i][0], h, source[i][1]]) *
                              plain.limited(old_scales[source[i][0], h, source[i][1] // 16]) for i in rows])
                s = plain.fitting(np.abs(v[np.isfinite(v)]).max(initial=0.0))
                kept = max(L - first, 0)
                if kept:
                    before = plain.limited(old_scales[p, h, r // 16])
                    s = max(s, before)
                    if s != before:
                        codes[p, h, r:r + kept] = plain.encode(plain.decode(codes[p, h, r:r + kept]) * (before / s))
                for i, x in zip(rows, v):
                    codes[p, h, r + L + i - first] = plain.encode(x / s)
                scales[p, h, r // 16] = s


@pytest.mark.parametrize("D,H_kv", [(128, 3), (64, 8)])
@pytest.mark.parametrize("L,gone", [(9, [1]), (9, [2]), (9, [1, 3]), (16, [2]), (30, [2]), (30, [1]), (30, [3, 4])])
@pytest.mark.parametrize("alias", [False, True])
def test_commit_without_some_pages(D, H_kv, L, gone, alias):
    """Drafts over several pages, some of the later ones missing, paths that cross a border of blocks."""
    N = 60
    for seed in range(4):
        rng, pk, pv, ks, vs, raw, scales, table = scaled_state(40 + seed, 2, H_kv, D, 16, [L, L], N)
        table[0, gone] = -1
        nodes = np.stack([np.sort(rng.choice(N, 14, replace=False)) for _ in range(2)]).astype(np.int32)
        n = np.array([14, 14 - seed], np.int32)
        kv = cuda(np.array([L, L], np.int32))
        rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, cuda(table), kv, cuda(nodes), cuda(n), N,
                                         new_kv_len=kv if alias else None)
        for i, (codes, sc) in enumerate(((pk, ks), (pv, vs))):
            plain_commit(raw[i], scales[i], table, [L, L], nodes, n, N)
            assert np.array_equal(sc.cpu().numpy(), scales[i]) and plain.same_codes(codes, raw[i])


@pytest.mark.parametrize("loud", [1, 6, 20])
def test_what_a_run_of_refused_drafts_costs(loud):
    """Drafts 2^loud louder than the accepted rows, all refused but their first node, which is as quiet as those: the block's
    scale grows to theirs and stays.  A row is off by half a step of its first code, 2^-4 of an element or 2^-10 of the
    scale, and by 2^-10 of every larger scale that it is rounded to later; those are powers of two, so in all by less than
    2^-4 of the element and 2^-9 of the last scale, which is no larger than the loudest draft needs."""
    rng, pk, pv, ks, vs, raw, scales, table = scaled_state(70, 1, 2, 64, 32, [32], 40)
    kv = cuda(np.array([32], np.int32))
    quiet = torch.from_numpy(rng.uniform(-1, 1, (1, 14, 2, 64))).to(BF16)
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), kv, quiet[:, :1].cuda(), quiet[:, :1].cuda())
    kv += 1
    grown = []
    for i in range(1, 14):
        draft = torch.from_numpy(rng.uniform(-1, 1, (1, 8, 2, 64)) * 2.0 ** loud).to(BF16)
        draft[:, 0] = quiet[:, i]
        rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, cuda(table), kv, draft.cuda(), draft.cuda())
        rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, cuda(table), kv, cuda(np.zeros((1, 1), np.int32)),
                                         cuda(np.ones(1, np.int32)), 8, new_kv_len=kv)
        p, _ = paged_util.row_of(table, 32, pk.shape[0], 0, 32)
        grown.append(ks[p, :, 0].cpu())
    scale = grown[-1].double()
    assert int(kv) == 46 and (scale <= plain.fitting(2.0 ** loud)).all() and (torch.stack(grown).diff(dim=0) >= 0).all()
    got = pk[p, :, :14].double().cpu() * scale[:, None, None]
    want = quiet[0].double().transpose(0, 1)
    assert ((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -9 * scale[:, None, None]).all()
