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
