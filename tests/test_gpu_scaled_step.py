"""The cache in codes as a serving loop uses it: a prompt appended, contexts forked, then steps of reserve -> append with
rotation -> attention -> acceptance -> commit -> release, eager and captured, held against the plain models."""
import math

import numpy as np
import pytest
import torch

import datagen
import paged_util
import paper_2311_08252_b200 as rest
import scaled_util as plain
from gpu_util import to_dev
from test_gpu_paged_attention_scaled import near

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def attention(q, codes, scales, table, kv_len, mask, N):
    k, v = (torch.from_numpy(plain.decode(codes[i])) *
            torch.from_numpy(scales[i]).double().repeat_interleave(16, 2)[..., None] for i in range(2))
    return paged_util.attention(q.cpu(), k, v, table, kv_len, mask, 1 / math.sqrt(q.shape[3]))


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("N,H", [(24, 4), (4, 6)])
def test_steps_over_codes(graph, N, H):
    rng = np.random.default_rng(5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    F, H_kv, D, page, cap, vocab, depth = 4, 2, 64, 16, 256, 300, 8
    P = 6 * cap // page
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    refs, table, n_pages, kv_len = i32(P), i32(F, cap // page).fill_(-1), i32(F), i32(F)
    pk, pv = (torch.full((P, H_kv, page, D), 0x7F, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    ks, vs = (torch.full((P, H_kv, page // 16), float("nan"), device="cuda") for _ in range(2))
    codes, scales = np.full((2, P, H_kv, page, D), 0x7F, np.uint8), np.full((2, P, H_kv, page // 16), np.nan, np.float32)
    freq, amplitude = rest.rotary_frequencies(D, scaling="parts", factor=4.0, original_len=128)
    turn = dict(inv_freq=freq.cuda(), amplitude=amplitude)
    spin = lambda x, pos: plain.turn(x.double().cpu().numpy(), pos, freq.numpy(), False, float(np.float32(amplitude)))  # noqa: E731

    # the prompts of contexts 0 and 1, then contexts 2 and 3 forked from them
    lens = to_dev(np.array([100, 37, 0, 0], np.int32))
    assert rest.rest_pages_reserve(refs, table, n_pages, lens, page).tolist() == [0] * F
    k, v = normal(F, 100, H_kv, D), normal(F, 100, H_kv, D)
    pos = torch.arange(100, dtype=torch.int32, device="cuda").expand(F, 100).contiguous()
    rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, table, kv_len, k, v, positions=pos, n_nodes=lens, **turn)
    for i, x in enumerate((spin(k, pos.cpu().numpy()), v.double().cpu().numpy())):
        plain.write(codes[i], scales[i], table.cpu().numpy(), [0] * F, x, lens.tolist())
    kv_len.copy_(lens)
    src, dst, st = rest.rest_pages_fork(refs, table, n_pages, kv_len, to_dev(np.array([1, 0], np.int32)),
                                        to_dev(np.array([2, 3], np.int32)), page)
    rest.rest_pages_copy_scaled(pk, pv, ks, vs, src, dst)
    for a, z in zip(src.tolist(), dst.tolist()):
        codes[:, z], scales[:, z] = codes[:, a], scales[:, a]
    assert st.tolist() == [0, 0]

    q, k, v = normal(F, N, H, D), normal(F, N, H_kv, D), normal(F, N, H_kv, D)
    mask, height, pos, turned = i32(F, N, 1), i32(F, N), i32(F, N), torch.zeros_like(q)
    tokens, parents, verifier = i32(F, N), i32(F, N), i32(F, N + 1)
    nodes, need, room = i32(F).fill_(N), i32(F), i32(F)
    out, lse = torch.zeros_like(q), torch.zeros((F, H, N), device="cuda")
    accepted = tuple(i32(*s) for s in ((F,), (F, depth), (F, depth + 1)))
    ws = torch.empty(rest.paged_attention_workspace_bytes(F, H, H_kv, N, D), dtype=torch.uint8, device="cuda")

    def step():
        torch.add(kv_len, N, out=need)
        torch.add(kv_len[:, None], height, out=pos)
        rest.rest_pages_reserve(refs, table, n_pages, need, page, status=room)
        rest.rest_paged_kv_append_scaled(pk, pv, ks, vs, table, kv_len, k, v, positions=pos, q=q, q_out=turned, **turn)
        rest.rest_paged_attention_scaled(turned, pk, pv, ks, vs, table, kv_len, mask, 1 / math.sqrt(D), out=out, lse=lse,
                                         workspace=ws)
        rest.rest_accept(tokens, parents, nodes, verifier, depth, out=accepted)
        rest.rest_paged_kv_commit_scaled(pk, pv, ks, vs, table, kv_len, accepted[1], accepted[0], N, new_kv_len=kv_len)
        rest.rest_pages_release(refs, table, n_pages, kv_len, page)

    if graph:
        state = [t.clone() for t in (refs, table, n_pages, kv_len, pk, pv, ks, vs)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t, s in zip((refs, table, n_pages, kv_len, pk, pv, ks, vs), state):
            t.copy_(s)
    total = 0
    for i in range(4):
        for t in (q, k, v):
            t.copy_(normal(*t.shape) * 2.0 ** float(rng.integers(-2, 3)))
        pa, dp, mk = zip(*(datagen.make_random_tree(100 * i + f, N, depth) for f in range(F)))
        tk = rng.permuted(np.tile(np.arange(vocab, dtype=np.int32), (F, 1)), axis=1)[:, :N]
        mk, pa = np.stack(mk).view(np.int32).reshape(F, N, 1), np.stack(pa)
        dp = np.array([[bin(int(w) & 0xFFFFFFFF).count("1") for w in row[:, 0]] for row in mk], np.int32)
        ver = rng.integers(0, vocab, (F, N + 1)).astype(np.int32)
        for f in range(F):                              # most nodes are what the verifier says after their parent
            for n in range(N):
                if rng.random() < 0.7:
                    ver[f, pa[f, n] + 1] = tk[f, n]
        for t, x in ((mask, mk), (height, dp - 1), (tokens, tk), (parents, pa), (verifier, ver)):
            t.copy_(to_dev(np.ascontiguousarray(x)))
        L = kv_len.cpu().numpy().copy()
        full, held = table.cpu().numpy().copy(), n_pages.cpu().numpy().copy()
        g.replay() if graph else step()
        torch.cuda.synchronize()
        at = L[:, None] + dp - 1
        assert room.tolist() == [0] * F and np.array_equal(pos.cpu().numpy(), at)
        # the draft's rows: pages that the step takes and may give back again
        free = [p for p in range(P) if p not in set(full[full >= 0].tolist())]
        for f in range(F):
            for c in range(held[f], -(-(int(L[f]) + N) // page)):
                full[f, c] = free.pop(0)
        for j, x in enumerate((spin(k, at), v.double().cpu().numpy())):
            plain.write(codes[j], scales[j], full, L, x, [N] * F)
        case = dict(q=turned, kv_len=L, vs=torch.from_numpy(scales[1]))
        near(case, out, lse, attention(turned, codes, scales, full, L, mk.view(np.uint32), N))
        n = accepted[0].cpu().numpy()
        for j in range(2):
            plain.commit(codes[j], scales[j], full, L, accepted[1].cpu().numpy(), n, N)
        total += int(n.sum())
        assert np.array_equal(kv_len.cpu().numpy(), L + n)
        for f in range(F):                              # rows in use, and their scales, to the bit
            rows = np.arange(int(L[f] + n[f]))
            for pool, sc, j in ((pk, ks, 0), (pv, vs, 1)):
                got = pool.view(torch.uint8)[table[f].long()[to_dev(rows) // page], :, to_dev(rows) % page].cpu().numpy()
                assert np.array_equal(got, codes[j][full[f][rows // page], :, rows % page])
                gs = sc[table[f].long()[to_dev(rows) // page], :, to_dev(rows) % page // 16].cpu().numpy()
                assert np.array_equal(gs, scales[j][full[f][rows // page], :, rows % page // 16])
    assert total > 6
    rest.rest_pages_release(refs, table, n_pages, torch.zeros_like(kv_len), page)
    assert int(refs.sum()) == 0


def test_calls_from_two_streams_with_scratch_of_their_own():
    B, N, H, D, page, L = 3, 40, 8, 128, 32, 900
    gen = torch.Generator(device="cuda").manual_seed(8)
    W = -(-(L + N) // page)
    cases = []
    for n in (N, 1):
        table = torch.randperm(B * W, generator=torch.Generator().manual_seed(3)).int().view(B, W).cuda()
        pool = [(torch.randn((B * W, 2, page, D), generator=gen, device="cuda") * 90).clamp(-448, 448).to(F8) for _ in range(2)]
        sc = [torch.rand((B * W, 2, page // 16), generator=gen, device="cuda") / 64 for _ in range(2)]
        cases.append((torch.randn((B, n, H, D), generator=gen, device="cuda").to(torch.bfloat16), *pool, *sc, table,
                      torch.full((B,), L, dtype=torch.int32, device="cuda"), None, 0.1))
    want = [rest.rest_paged_attention_scaled(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(20):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append(rest.rest_paged_attention_scaled(*c))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)
