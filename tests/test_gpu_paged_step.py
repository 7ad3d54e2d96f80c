"""The paged operators together, as a serving loop uses them: contexts forked, then steps of reserve ->
write -> attention -> acceptance -> commit -> release, held against contiguous caches, the contiguous
attention call and the greedy acceptance that the library has besides."""
import math

import numpy as np
import pytest
import torch

import datagen
import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("graph", [False, True])
def test_steps_over_pages_equal_steps_over_contiguous_caches(graph):
    rng = np.random.default_rng(5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    B, F, N, H, D, page, cap, vocab, depth = 2, 4, 24, 4, 128, 16, 512, 300, 8
    P = 6 * cap // page
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    table = torch.full((F, cap // page), -1, dtype=torch.int32, device="cuda")
    n_pages, kv_len = (torch.zeros(F, dtype=torch.int32, device="cuda") for _ in range(2))
    pk, pv = (torch.full((P, H, page, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ck, cv = (torch.zeros((F, H, cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    # prompts of contexts 0 and 1, then contexts 2 and 3 forked from them
    lens = to_dev(np.array([100, 37, 0, 0], np.int32))
    assert rest.rest_pages_reserve(refs, table, n_pages, lens, page).tolist() == [0] * F
    k, v = normal(F, 128, H, D), normal(F, 128, H, D)
    rest.rest_paged_kv_write(pk, pv, table, kv_len, k, v, n_nodes=lens)
    kv_len.copy_(lens)
    for f, src in enumerate((0, 1, 1, 0)):
        for c, new in ((ck, k), (cv, v)):
            c[f, :, :128] = new[src].transpose(0, 1)
    src, dst, st = rest.rest_pages_fork(refs, table, n_pages, kv_len, to_dev(np.array([1, 0], np.int32)),
                                        to_dev(np.array([2, 3], np.int32)), page)
    rest.rest_pages_copy(pk, pv, src, dst)
    assert st.tolist() == [0, 0] and kv_len.tolist() == [100, 37, 37, 100]
    flat_len = kv_len.clone()

    # buffers of one step, so that it can be captured
    q, k, v = normal(F, N, H, D), normal(F, N, H, D), normal(F, N, H, D)
    mask = torch.zeros((F, N, 1), dtype=torch.int32, device="cuda")
    tokens, parents = (torch.zeros((F, N), dtype=torch.int32, device="cuda") for _ in range(2))
    nodes = torch.full((F,), N, dtype=torch.int32, device="cuda")
    logits, uni = normal(F, N + 1, vocab), torch.rand((F, N + 1), generator=gen, device="cuda")
    temp, top_p = torch.zeros(F, device="cuda"), torch.ones(F, device="cuda")
    out = torch.zeros_like(q)
    accepted = tuple(torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((F,), (F, depth), (F, depth + 1)))
    need, room = torch.zeros_like(kv_len), torch.zeros_like(kv_len)
    ws = torch.empty(rest.paged_attention_workspace_bytes(F, H, H, N, D), dtype=torch.uint8, device="cuda")
    scale = 1 / math.sqrt(D)

    def step():
        torch.add(kv_len, N, out=need)
        rest.rest_pages_reserve(refs, table, n_pages, need, page, status=room)
        rest.rest_paged_kv_write(pk, pv, table, kv_len, k, v)
        rest.rest_paged_attention(q, pk, pv, table, kv_len, mask, scale, out=out, workspace=ws)
        rest.rest_accept_sampled(logits, tokens, parents, nodes, uni, temp, top_p, depth, out=accepted, workspace=False)
        rest.rest_paged_kv_commit(pk, pv, table, kv_len, accepted[1], accepted[0], N, new_kv_len=kv_len)
        rest.rest_pages_release(refs, table, n_pages, kv_len, page)

    if graph:
        state = [t.clone() for t in (refs, table, n_pages, kv_len, pk, pv)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t, s in zip((refs, table, n_pages, kv_len, pk, pv), state):
            t.copy_(s)
    total = 0
    for i in range(6):
        for t in (q, k, v):
            t.copy_(normal(*t.shape))
        pa, _, mk = zip(*(datagen.make_random_tree(100 * i + f, N, depth) for f in range(F)))
        tk = rng.permuted(np.tile(np.arange(vocab, dtype=np.int32), (F, 1)), axis=1)[:, :N]
        mask.copy_(to_dev(np.stack(mk).view(np.int32).reshape(F, N, 1)))
        tokens.copy_(to_dev(tk)), parents.copy_(to_dev(np.stack(pa)))
        lg = normal(F, N + 1, vocab).float()
        for f in range(F):                                       # most nodes are what their parent's row says
            for n in range(N):
                if rng.random() < 0.7:
                    lg[f, int(pa[f][n]) + 1, int(tk[f][n])] = 8 + n / 8
        logits.copy_(lg)
        g.replay() if graph else step()

        # the same over contiguous caches
        for f in range(F):
            L = int(flat_len[f])
            for c, new in ((ck, k), (cv, v)):
                c[f, :, L:L + N] = new[f].transpose(0, 1)
        want = rest.rest_tree_attention(q, ck, cv, flat_len, mask, scale)
        # each is within 2^-8 (|out| + A) + 2^-15 (S + 1) A of 64 bits; |out| <= A < 2 and S < 16 here
        assert (out.float() - want.float()).abs().max() <= 2 * (4 * 2.0 ** -8 + 2 * 17 * 2.0 ** -15), i
        acc = rest.rest_accept(tokens, parents, nodes, logits.float().argmax(-1).int(), depth)
        for a, b in zip(accepted, acc):
            assert torch.equal(a, b)
        rest.rest_kv_commit(ck, cv, flat_len, acc[1], acc[0], N, new_kv_len=flat_len)
        assert torch.equal(kv_len, flat_len) and room.tolist() == [0] * F
        total += int(acc[0].sum())
        # what the pages hold is what the contiguous caches hold, and shared pages stay shared
        for f in range(F):
            L = int(flat_len[f])
            rows = torch.arange(L, device="cuda")
            for pool, c in ((pk, ck), (pv, cv)):
                assert torch.equal(pool[table[f].long()[rows // page], :, rows % page], c[f, :, :L].transpose(0, 1))
        assert table[0, 5] == table[3, 5] and refs[table[0, 5].long()] == 2
        assert int((refs > 0).sum()) == len(set(table[table >= 0].tolist()))
    assert total > 10
    rest.rest_pages_release(refs, table, n_pages, torch.zeros_like(kv_len), page)
    assert int(refs.sum()) == 0


def test_calls_from_two_streams_with_scratch_of_their_own():
    B, N, H, D, page, L = 3, 8, 8, 128, 32, 900
    gen = torch.Generator(device="cuda").manual_seed(8)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    W = -(-(L + N) // page)
    cases = []
    for _ in range(2):
        table = torch.randperm(B * W, generator=torch.Generator().manual_seed(3)).int().view(B, W).cuda()
        cases.append((normal(B, N, H, D), normal(B * W, 2, page, D), normal(B * W, 2, page, D), table,
                      torch.full((B,), L, dtype=torch.int32, device="cuda"), None, 0.1))
    want = [rest.rest_paged_attention(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(20):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append(rest.rest_paged_attention(*c))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)
