"""A plain model of a cache in pages (numpy and Python loops) that the kernels are held to."""
import numpy as np


def row_of(table, page, P, b, at):
    """(page, row) of row `at` of context b, or None when the table has no such page."""
    col = at // page
    if at < 0 or col >= table.shape[1] or not 0 <= table[b, col] < P:
        return None
    return int(table[b, col]), at % page


def write(pool, table, kv_len, new, n_nodes=None):
    P, _, page, _ = pool.shape
    B, N = new.shape[:2]
    for b in range(B):
        for i in range(N if n_nodes is None else min(N, int(n_nodes[b]))):
            at = row_of(table, page, P, b, int(kv_len[b]) + i) if kv_len[b] >= 0 else None
            if at:
                pool[at[0], :, at[1]] = new[b, i]


def commit(pool, table, kv_len, nodes, lens, N):
    P, _, page, _ = pool.shape
    old = pool.copy()
    for b in range(len(kv_len)):
        for i in range(min(max(int(lens[b]), 0), nodes.shape[1])):
            nd = min(max(int(nodes[b, i]), 0), N - 1)
            frm, to = row_of(table, page, P, b, int(kv_len[b]) + nd), row_of(table, page, P, b, int(kv_len[b]) + i)
            if frm and to and kv_len[b] >= 0:
                pool[to[0], :, to[1]] = old[frm[0], :, frm[1]]


def fork(refs, table, n_pages, kv_len, parents, children, page):
    """In place; returns (copy_src, copy_dst, status)."""
    P, B = len(refs), len(n_pages)
    entry = refs.copy(), table.copy(), n_pages.copy(), kv_len.copy()
    free = [p for p in range(P) if entry[0][p] == 0]
    src, dst, status, seen = [], [], [], set()
    taken = 0
    for pa, ch in zip(parents.tolist(), children.tolist()):
        a = z = -1
        st = 0
        if not (0 <= ch < B and 0 <= pa < B) or pa == ch or entry[2][ch] != 0 or ch in seen:
            st = 5
        seen.add(ch)
        L = 0
        if st == 0 and entry[2][pa] != 0:
            L = int(entry[3][pa])
            if L < 0 or -(-L // page) > min(entry[2][pa], table.shape[1]):
                st = 5
        full, part = L // page, int(L % page != 0)
        if st == 0 and part:
            if taken >= len(free):
                st = 4
            taken += 1
        if st == 0:
            table[ch] = -1
            for c in range(full):
                p = int(entry[1][pa, c])
                if 0 <= p < P:
                    table[ch, c] = p
                    refs[p] += 1
            if part:
                a, z = int(entry[1][pa, full]), free[taken - 1]
                a = a if 0 <= a < P else -1
                table[ch, full] = z
                refs[z] = 1
            n_pages[ch], kv_len[ch] = full + part, L
        src.append(a), dst.append(z), status.append(st)
    return tuple(np.array(x, np.int32) for x in (src, dst, status))


def reserve(refs, table, n_pages, need_len, page):
    free = [p for p in range(len(refs)) if refs[p] == 0]
    asked, status = 0, []
    for b in range(len(n_pages)):
        have, want = int(n_pages[b]), -(-max(int(need_len[b]), 0) // page)
        if not 0 <= have <= table.shape[1] or want > table.shape[1]:
            status.append(5)
            continue
        need = max(want - have, 0)
        first, asked = asked, asked + need
        if need and asked > len(free):
            status.append(4)
            continue
        for j in range(need):
            table[b, have + j] = free[first + j]
            refs[free[first + j]] = 1
        n_pages[b] = have + need
        status.append(0)
    return np.array(status, np.int32)


def release(refs, table, n_pages, keep_len, page, window=0, sinks=0):
    for b in range(len(n_pages)):
        keep = int(keep_len[b])
        if keep < 0:
            continue
        kept = -(-keep // page)
        for c in range(int(n_pages[b])):
            first, last = c * page, (c + 1) * page - 1
            if c < kept and not (window > 0 and first >= sinks and last <= keep - window):
                continue
            p = int(table[b, c])
            table[b, c] = -1
            if 0 <= p < len(refs) and refs[p] > 0:
                refs[p] -= 1
        n_pages[b] = min(int(n_pages[b]), kept)


def attention(q, k, v, table, kv_len, mask, scale, window=0, sinks=0, n_nodes=None):
    """softmax(scale q.k) v over the visible keys in 64 bits (torch tensors on the CPU, pages
    [P,H_kv,page,D]).  Returns (out [B,N,H,D], lse [B,H,N], A, S): A = sum p |v| and S = the largest
    scale * sum |q k| of each row, which error bounds are made of.  Rows past n_nodes are NaN."""
    import torch
    B, N, H, D = q.shape
    P, H_kv, page, _ = k.shape
    out = torch.full((B, N, H, D), float("nan"), dtype=torch.float64)
    A, lse = out.clone(), torch.full((B, H, N), float("nan"), dtype=torch.float64)
    S = torch.zeros((B, H, N), dtype=torch.float64)
    for b in range(B):
        L, n = int(kv_len[b]), N if n_nodes is None else int(n_nodes[b])
        if n == 0:
            continue
        sees = torch.zeros((n, L + n), dtype=torch.bool)
        sees[:, :L] = True
        for i in range(n):
            for j in range(n):
                sees[i, L + j] = j <= i if mask is None else bool((int(mask[b, i, j >> 5]) >> (j & 31)) & 1)
        depth = (np.arange(N) + 1 if mask is None else
                 np.array([sum(bin(int(w) & 0xFFFFFFFF).count("1") for w in mask[b, i]) for i in range(N)]))
        at = torch.tensor(list(range(L)) + [L + max(int(depth[j]), 1) - 1 for j in range(n)])
        if window:
            sees &= (at[None] < sinks) | (at[None] > at[L:, None] - window)
        keys = [row_of(table, page, P, b, r) for r in range(L + n)]
        K = torch.stack([k[p[0], :, p[1]].double() if p else torch.zeros((H_kv, D), dtype=torch.float64) for p in keys])
        V = torch.stack([v[p[0], :, p[1]].double() if p else torch.zeros((H_kv, D), dtype=torch.float64) for p in keys])
        for h in range(H):
            kk, vv, qq = K[:, h // (H // H_kv)], V[:, h // (H // H_kv)], q[b, :n, h].double()
            for i in range(n):
                on = sees[i].nonzero()[:, 0]
                if len(on) == 0:
                    out[b, i, h], A[b, i, h], lse[b, h, i] = 0.0, 0.0, -float("inf")
                    continue
                x = scale * (kk[on] @ qq[i])
                p = torch.softmax(x, 0)
                out[b, i, h], A[b, i, h] = p @ vv[on], p @ vv[on].abs()
                lse[b, h, i] = torch.logsumexp(x, 0)
                S[b, h, i] = scale * (kk[on].abs() @ qq[i].abs()).max()
    return out, lse, A, S


def assert_attention(got, got_lse, ref, dtype, n_keys):
    """Every element within what its roundings allow.  With e = half a step of the type (2^-8 bf16,
    2^-11 fp16): the output's rounding e |out|; the probabilities' rounding e A, and for fp16 half of
    its smallest step (2^-25 of the largest) for each key; scores in 32 bits, 128 products added in any
    order, the scale and the exponential: 2^-16 (S + 1) relative for each probability and for their
    sum, so 2 * 2^-16 (S + 1) A.  lse: 2^-16 (S + 1), and 2^-22 of its value for log and product."""
    import torch
    out, lse, A, S = ref
    e = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    rel = (S + 1).transpose(1, 2)[..., None] * 2.0 ** -15
    tol = e * out.abs() + (e + rel) * A * (1 + e) + (0 if dtype == torch.bfloat16 else n_keys * 2.0 ** -25 * 8) + 1e-30
    got, live = got.double().cpu(), ~out.isnan()
    over = ((got - out).abs() - tol)[live]
    assert not got[live].isnan().any() and over.max() <= 0, float(over.max())
    if got_lse is not None:
        g, w = got_lse.double().cpu(), lse
        seen = w.isfinite()
        assert torch.equal(g[w.isinf()], w[w.isinf()])
        if seen.any():
            over = ((g - w).abs() - (S + 1) * 2.0 ** -16 - w.abs() * 2.0 ** -22)[seen]
            assert over.max() <= 0, float(over.max())


def accept_sampled(logits, tokens, parents, n_nodes, uniforms, temperature, top_p, max_depth):
    """The acceptance walk in 64 bits (numpy; logits float64 [B,N+1,V])."""
    B, N = tokens.shape
    V = logits.shape[2]
    lens, nodes, out = np.zeros(B, np.int32), np.full((B, max_depth), -1, np.int32), np.full((B, max_depth + 1), -1, np.int32)
    for b in range(B):
        cur, n = -1, 0
        u = np.clip(np.nan_to_num(uniforms[b].astype(np.float64), nan=0.0), 0.0, np.float64(np.float32(0.99999994)))
        while True:
            x = logits[b, cur + 1].astype(np.float64).copy()
            x[np.isnan(x)] = -np.inf
            if not (x > -np.inf).any():
                break                                              # nothing can be drawn: -1
            order = np.lexsort((np.arange(V), -x))
            w = np.zeros(V)
            if temperature[b] > 0:
                with np.errstate(invalid="ignore", over="ignore"):
                    w = np.where(x == x.max(), 1.0, np.exp((x - x.max()) / np.float64(temperature[b])))
                w[w < 2.0 ** -44] = 0.0
                if top_p[b] < 1:
                    before = np.cumsum(w[order]) - w[order]
                    drop = before >= np.float64(top_p[b]) * w.sum()
                    drop[0] = False
                    w[order[drop]] = 0.0
            else:
                w[order[0]] = 1.0
            child = -1
            for c in range(min(max(int(n_nodes[b]), 0), N)):
                if n < max_depth and parents[b, c] == cur and 0 <= tokens[b, c] < V and w[tokens[b, c]] > 0:
                    if u[c + 1] * w.sum() < w[tokens[b, c]]:
                        child = c
                        break
                    w[tokens[b, c]] = 0.0
            if child < 0:
                cdf = np.cumsum(w)
                out[b, n] = int(np.argmax(cdf > u[0] * cdf[-1]))
                break
            nodes[b, n], out[b, n] = child, tokens[b, child]
            n, cur = n + 1, child
        lens[b] = n
    return lens, nodes, out
