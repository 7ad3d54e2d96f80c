"""The serving operators around the draft tree, as measurable cases.

    attn    rest_paged_attention: draft rows (or single tokens) over a paged KV cache, with an
            optional sliding window and first tokens that stay visible
    accept  rest_accept_sampled: acceptance of a draft tree against the target's probabilities
    rows    rest_paged_kv_write, rest_paged_kv_commit: a step's new K/V rows into the pages, then
            the accepted path moved to the front
    fork    rest_pages_fork, rest_pages_copy, rest_pages_reserve, rest_pages_release: contexts
            forked, room for the next rows, pages behind the window given back

`own = False` computes them with elementary torch operations, `own = True` through the package."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one token of one stream: latency
        dict(name="attn_token_b1", op="attn", B=1, N=1, H=32, Hkv=8, D=128, page=16, L=2048, ragged=False,
             window=0, sinks=0, dtype="bf16"),
        # the single-stream draft tree of a model with one KV head per query head
        dict(name="attn_tree_b1", op="attn", B=1, N=64, H=32, Hkv=32, D=128, page=64, L=2048, ragged=False,
             window=0, sinks=0, dtype="bf16"),
        # a serving batch of draft trees, uneven prefixes and trees, grouped KV heads, small pages
        dict(name="attn_tree_batch", op="attn", B=61, N=64, H=32, Hkv=8, D=128, page=16, L=4096, ragged=True,
             window=0, sinks=0, dtype="bf16"),
        # large trees over long prefixes, five query heads per KV head
        dict(name="attn_tree_long", op="attn", B=16, N=128, H=40, Hkv=8, D=128, page=64, L=16384, ragged=False,
             window=0, sinks=0, dtype="bf16"),
        # draft trees of a model with a sliding window: pages behind it are gone
        dict(name="attn_tree_window", op="attn", B=64, N=33, H=32, Hkv=8, D=128, page=32, L=16384, ragged=True,
             window=4096, sinks=4, dtype="bf16"),
        # ordinary decoding of a large batch of small heads under a window
        dict(name="attn_tokens_window", op="attn", B=256, N=1, H=32, Hkv=8, D=64, page=128, L=8192, ragged=True,
             window=2048, sinks=64, dtype="fp16"),
        # sampled acceptance for one stream, and for a batch
        dict(name="accept_b1", op="accept", B=1, N=64, V=32000, max_depth=10, dtype="bf16", temperature=0.8,
             top_p=0.95),
        dict(name="accept_batch", op="accept", B=128, N=64, V=32000, max_depth=16, dtype="fp32", temperature=0.8,
             top_p=0.95),
        # one layer's cache rows of one step: one stream, and a batch
        dict(name="rows_b1", op="rows", B=1, N=64, Hkv=32, D=128, page=16, L=2048, max_depth=10, dtype="bf16"),
        dict(name="rows_batch", op="rows", B=128, N=64, Hkv=32, D=128, page=64, L=1024, max_depth=16, dtype="bf16"),
        # a prompt's context forked into a few samples, and a batch of them
        dict(name="fork_few", op="fork", contexts=1, each=3, N=64, Hkv=8, D=128, page=16, L=2048, window=0, sinks=0,
             dtype="bf16"),
        dict(name="fork_many", op="fork", contexts=64, each=7, N=64, Hkv=8, D=128, page=128, L=4096, window=1024,
             sinks=4, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "accept", "rows", "fork"])
    dtype = rng.choice(["bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    D = rng.choice([64, 128])
    window = rng.choice([0, _log(rng, 40, 5000)])
    sinks = rng.choice([0, 4, rng.randint(1, 200)]) if window else 0
    if op == "attn":
        Hkv, G, N = rng.choice([1, 2, 4, 8]), rng.choice([1, 3, 4, 5, 8]), rng.choice([1, _log(rng, 1, 256)])
        L = _log(rng, 1, 16384)
        seen = (min(L, window + sinks) if window else L) + N
        most = min(256, int(2.5e8 / (Hkv * seen * D)), int(2.5e11 / (Hkv * G * N * seen * D * 4)),
                   int(1.3e9 / (Hkv * G * N * (L + N))), int(1e9 / (Hkv * (L + N) * D)))
        return dict(op=op, B=_log(rng, 1, max(1, most)), N=N, H=Hkv * G, Hkv=Hkv, D=D, page=page, L=L,
                    ragged=rng.random() < 0.7, window=window, sinks=sinks, dtype=dtype)
    if op == "accept":
        V, N = _log(rng, 1000, 130000), _log(rng, 1, 256)
        most = min(128, int(2.6e8 / ((N + 1) * V)))
        return dict(op=op, B=_log(rng, 1, max(1, most)), N=N, V=V, max_depth=rng.randint(1, 16),
                    dtype=rng.choice(["bf16", "fp16", "fp32"]), temperature=rng.choice([0.0, 0.6, 0.8, 1.0, 1.3]),
                    top_p=rng.choice([0.5, 0.9, 0.95, 1.0]))
    if op == "rows":
        return dict(op=op, B=_log(rng, 1, 128), N=_log(rng, 1, 64), Hkv=rng.choice([1, 4, 8, 32]), D=D, page=page,
                    L=_log(rng, 1, 1024), max_depth=rng.randint(1, 16), dtype=dtype)
    return dict(op=op, contexts=_log(rng, 1, 64), each=rng.randint(1, 7), N=_log(rng, 1, 64), Hkv=rng.choice([1, 4, 8]),
                D=D, page=page, L=_log(rng, 1, 4096), window=window, sinks=sinks, dtype=dtype)


# ---------------------------------------------------------------------------------------- inputs
def _trees(rng, B, N, max_depth, n_nodes):
    """Random trees: parents int32[B,N] (-1: child of the root), depth, packed ancestor masks."""
    parents = np.full((B, N), -1, np.int64)
    depth = np.ones((B, N), np.int64)
    seen = np.zeros((B, N, N), bool)
    rows = np.arange(B)
    for i in range(N):
        p = rng.integers(-1, i, B) if i else np.full(B, -1)
        p = np.where((p >= 0) & (depth[rows, p] >= max_depth), parents[rows, p], p)
        p = np.where(i < n_nodes, p, -1)
        parents[:, i] = p
        has = p >= 0
        depth[:, i] = np.where(has, depth[rows, p] + 1, 1)
        seen[:, i] = seen[rows, p] & has[:, None]
        seen[:, i, i] = True
    packed = np.zeros((B, N, (N + 31) // 32 * 32), np.uint8)
    packed[:, :, :N] = seen
    words = np.packbits(packed.reshape(B, N, -1, 32), axis=-1, bitorder="little").view(np.uint32).reshape(B, N, -1)
    return parents.astype(np.int32), depth, seen, words.view(np.int32).copy()


def _tables(rng, lens, new, most, page, window, sinks, spare):
    """Block tables of contexts with lens[b] rows and room for `new` more (`most` rows in all at
    most), pages in random order; pages wholly behind the window are gone (-1)."""
    B = len(lens)
    want = -(-(lens + new) // page)
    W = int(want.max())
    col = np.arange(W)[None]
    held = col < want[:, None]
    if window:
        held &= ~((col * page >= sinks) & ((col + 1) * page - 1 <= (lens - window)[:, None]))
    n = B * -(-most // page)                               # the pool's size goes by the case alone
    table = np.full((B, W), -1, np.int32)
    table[held] = rng.permutation(n)[:int(held.sum())]
    return table, n + spare


def prepare(case, seed):
    dev = torch.device("cuda")
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    to = lambda a, t=None: torch.from_numpy(np.ascontiguousarray(a)).to(dev, t)  # noqa: E731
    normal = lambda *shape: torch.empty(shape, dtype=dt, device=dev).normal_(generator=gen)  # noqa: E731
    st = dict(case=dict(case))
    op = case["op"]
    if op == "attn":
        B, N, H, Hkv, D, L = (case[k] for k in ("B", "N", "H", "Hkv", "D", "L"))
        lens = rng.integers(L // 2, L + 1, B) if case["ragged"] else np.full(B, L)
        nodes = rng.integers((N + 1) // 2, N + 1, B) if case["ragged"] else np.full(B, N)
        parents, depth, seen, words = _trees(rng, B, N, 10, nodes)
        table, P = _tables(rng, lens, N, min(L, case["window"] + case["sinks"] + 3 * case["page"] if case["window"] else L) + N,
                           case["page"], case["window"], case["sinks"], 1)
        # some heads look at their keys more sharply than others
        sharp = torch.linspace(0.5, 2.0, H, device=dev)[None, None, :, None]
        st.update(q=(normal(B, N, H, D).float() * sharp).to(dt), k=normal(P, Hkv, case["page"], D),
                  v=normal(P, Hkv, case["page"], D), table=to(table), kv_len=to(lens, torch.int32),
                  n_nodes=to(nodes, torch.int32), mask=to(words), out=torch.zeros((B, N, H, D), dtype=dt, device=dev),
                  lse=torch.zeros((B, H, N), dtype=torch.float32, device=dev), depth=to(depth), seen=to(seen))
    elif op == "accept":
        B, N, V = case["B"], case["N"], case["V"]
        nodes = rng.integers((N + 1) // 2, N + 1, B)
        parents, depth, seen, words = _trees(rng, B, N, case["max_depth"], nodes)
        tokens = rng.integers(0, V, (B, N)).astype(np.int32)
        logits = torch.empty((B, N + 1, V), dtype=torch.float32, device=dev).normal_(generator=gen).mul_(2.0)
        # drafted tokens are likely ones: each weighs about as much as all others of its row
        peak = to(rng.normal(math.log(V) + 2.0, 1.0, (B, N)), torch.float32)
        b = torch.arange(B, device=dev)[:, None].expand(B, N)
        logits[b, to(parents).long() + 1, to(tokens).long()] = peak
        st.update(logits=logits.to(dt), tokens=to(tokens), parents=to(parents), n_nodes=to(nodes, torch.int32),
                  uniforms=torch.rand((B, N + 1), generator=gen, device=dev),
                  temperature=torch.full((B,), case["temperature"], device=dev),
                  top_p=torch.full((B,), case["top_p"], device=dev))
    elif op == "rows":
        B, N, Hkv, D = case["B"], case["N"], case["Hkv"], case["D"]
        lens = rng.integers(case["L"] // 2, case["L"] + 1, B)
        nodes = rng.integers((N + 1) // 2, N + 1, B)
        parents, depth, seen, words = _trees(rng, B, N, case["max_depth"], nodes)
        table, P = _tables(rng, lens, N, case["L"] + N, case["page"], 0, 0, 1)
        # the accepted path: a random node's, from the root
        leaf = rng.integers(0, nodes)
        path = np.full((B, case["max_depth"]), -1, np.int32)
        on = seen[np.arange(B), leaf]
        rank = np.cumsum(on, 1) - 1
        bb, nn = np.nonzero(on)
        path[bb, rank[bb, nn]] = nn
        st.update(k=normal(P, Hkv, case["page"], D), v=normal(P, Hkv, case["page"], D), table=to(table),
                  kv_len=to(lens, torch.int32), n_nodes=to(nodes, torch.int32), k_new=normal(B, N, Hkv, D),
                  v_new=normal(B, N, Hkv, D), accept_nodes=to(path), accept_len=to(on.sum(1), torch.int32),
                  new_kv_len=torch.zeros(B, dtype=torch.int32, device=dev))
    else:
        C, F, page = case["contexts"], case["contexts"] * case["each"], case["page"]
        lens = rng.integers(case["L"] // 2, case["L"] + 1, C)
        W = -(-(case["L"] + case["N"] + 1) // page)
        held, n = _tables(rng, lens, 0, case["L"], page, case["window"], case["sinks"], 0)
        P = n + F + (C + F) * -(-case["N"] // page) + 8
        where = rng.permutation(P).astype(np.int32)
        table = np.full((C + F, W), -1, np.int32)
        w = min(W, held.shape[1])
        table[:C, :w] = np.where(held[:, :w] >= 0, where[held[:, :w]], -1)
        refs = np.zeros(P + 1, np.int32)
        refs[table[table >= 0]] = 1
        refs[P] = 1                                  # the last page is never given out
        n_pages = np.zeros(C + F, np.int32)
        n_pages[:C] = -(-lens // page)
        kv_len = np.zeros(C + F, np.int32)
        kv_len[:C] = lens
        st.update(k=normal(P + 1, case["Hkv"], page, case["D"]), v=normal(P + 1, case["Hkv"], page, case["D"]),
                  refs=to(refs), table=to(table), n_pages=to(n_pages), kv_len=to(kv_len),
                  parent=to(np.repeat(np.arange(C), case["each"]).astype(np.int32)),
                  child=to(np.arange(C, C + F).astype(np.int32)))
    return st


# ------------------------------------------------------------------------------------ plain forms
def _plain_attn(s):
    c = s["case"]
    B, N, H, Hkv, D, page = (c[k] for k in ("B", "N", "H", "Hkv", "D", "page"))
    G, W = H // Hkv, s["table"].shape[1]
    T = W * page
    rows = s["table"].clamp(min=0).long()
    k = s["k"][rows].permute(0, 2, 1, 3, 4).reshape(B, Hkv, T, D).float()
    v = s["v"][rows].permute(0, 2, 1, 3, 4).reshape(B, Hkv, T, D).float()
    q = s["q"].view(B, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, D).float()
    L, nodes = s["kv_len"].long()[:, None, None], s["n_nodes"].long()[:, None, None]
    key = torch.arange(T, device=q.device)[None, None]
    bit = torch.arange(N, device=q.device)
    tree = ((s["mask"][:, :, bit >> 5] >> (bit & 31)) & 1).bool()                 # [B,N,N]
    depth = tree.sum(-1)                                                          # [B,N]
    node = (key - L).clamp(0, N - 1)                                              # [B,1,T]
    in_tree = (key >= L) & (key < L + nodes)
    seen = (key < L) | (in_tree & tree.gather(2, node.expand(B, N, T)))
    if c["window"]:
        at = torch.where(key < L, key, L + depth.gather(1, node[:, 0])[:, None] - 1)   # position of a key
        seen &= (at < c["sinks"]) | (at > L + depth[:, :, None] - 1 - c["window"])
    score = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, G, N, T)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e.div_(total).view(B, Hkv, G * N, T) @ v).view(B, Hkv, G, N, D)
    live = (torch.arange(N, device=q.device)[None] < s["n_nodes"][:, None])       # rows past the tree stay 0
    o = o.permute(0, 3, 1, 2, 4).reshape(B, N, H, D) * live[:, :, None, None]
    lse = (top + total.log()).view(B, H, N) * live[:, None]
    return {"out": o.to(s["q"].dtype), "lse": lse}


def _plain_accept(s):
    c = s["case"]
    B, N, V, depth = c["B"], c["N"], c["V"], c["max_depth"]
    dev = s["logits"].device
    every = torch.arange(B, device=dev)
    slot = torch.arange(N, device=dev)[None]
    tokens, u = s["tokens"].long(), s["uniforms"].double()
    earlier = torch.tril(torch.ones((N, N), dtype=torch.bool, device=dev), -1)
    cur = torch.full((B,), -1, dtype=torch.long, device=dev)
    length = torch.zeros(B, dtype=torch.long, device=dev)
    nodes = torch.full((B, depth), -1, dtype=torch.int32, device=dev)
    out = torch.full((B, depth + 1), -1, dtype=torch.int32, device=dev)
    alive = torch.ones(B, dtype=torch.bool, device=dev)
    for step in range(depth + 1):
        x = s["logits"][every, cur + 1].double()
        top = x.amax(1, keepdim=True)
        if c["temperature"] == 0.0:
            p = torch.zeros_like(x)
            p[every, x.argmax(1)] = 1.0
        else:
            p = ((x - top) / s["temperature"].double()[:, None]).exp()
            p = p / p.sum(1, keepdim=True)
            order = x.sort(dim=1, descending=True, stable=True).indices
            ranked = p.gather(1, order)
            before = ranked.cumsum(1) - ranked
            keep = before < s["top_p"].double()[:, None]
            p = p * torch.zeros_like(keep).scatter_(1, order, keep)
            p = p / p.sum(1, keepdim=True)
        child = (s["parents"] == cur[:, None]) & (slot < s["n_nodes"][:, None]) & (step < depth)
        again = (tokens[:, :, None] == tokens[:, None, :]) & child[:, None, :] & earlier[None]
        pc = p.gather(1, tokens) * child * ~again.any(2)
        left = 1.0 - (pc.cumsum(1) - pc)
        yes = child & (u[:, 1:] * left < pc)
        hit, first = yes.any(1), yes.to(torch.int8).argmax(1)
        # nothing accepted: a token from what the refused children leave
        p = p.masked_fill(torch.zeros_like(p).scatter_add_(1, tokens, child.double()) > 0, 0.0)
        cdf = p.cumsum(1)
        drawn = (cdf <= u[:, :1] * cdf[:, -1:]).sum(1).clamp(max=V - 1)
        go, stop = alive & hit, alive & ~hit
        if step < depth:
            nodes[:, step] = torch.where(go, first.int(), nodes[:, step])
        out[:, step] = torch.where(go, tokens.gather(1, first[:, None])[:, 0].int(),
                                   torch.where(stop, drawn.int(), out[:, step]))
        length = length + go
        cur = torch.where(go, first, cur)
        alive = go
    return {"len": length.int(), "nodes": nodes, "tokens": out}


def _plain_rows(s):
    N, page = s["case"]["N"], s["case"]["page"]
    b = torch.arange(s["case"]["B"], device=s["k"].device)[:, None]
    L = s["kv_len"].long()[:, None]
    i = torch.arange(N, device=b.device)[None]
    j = torch.arange(s["case"]["max_depth"], device=b.device)[None]
    at = L + i
    pg, row = s["table"][b, at // page].long(), at % page
    new = (i < s["n_nodes"][:, None])[:, :, None, None]
    to_at = L + j
    fits = s["table"].shape[1] - 1
    moved = j < s["accept_len"][:, None]
    from_at = torch.where(moved, L + s["accept_nodes"].long(), to_at)
    spare = s["k"].shape[0] - 1                            # where nothing moves, the spare page is read and written
    p0 = torch.where(moved, s["table"][b, (from_at // page).clamp(max=fits)].long(), spare)
    p1 = torch.where(moved, s["table"][b, (to_at // page).clamp(max=fits)].long(), spare)
    r0, r1 = torch.where(moved, from_at % page, 0), torch.where(moved, to_at % page, 0)
    got = []
    for pool, fresh in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        pool[pg, :, row] = torch.where(new, fresh, pool[pg, :, row])
        pool[p1, :, r1] = pool[p0, :, r0]
        got.append(pool)
    return {"k": got[0], "v": got[1], "kv_len": (s["kv_len"] + s["accept_len"]).int()}


def _plain_take(refs, need):
    """need[f] free pages for each f in turn, lowest numbers first: exclusive offsets, whether they
    can be had, and the free pages in order."""
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices
    upto = need.cumsum(0)
    return upto - need, upto <= (refs == 0).sum(), free


def _plain_fork(s):
    c = s["case"]
    page, P = c["page"], s["refs"].shape[0]
    refs, table, n_pages, kv_len = s["refs"].clone(), s["table"].clone(), s["n_pages"].clone(), s["kv_len"].clone()
    par, ch = s["parent"].long(), s["child"].long()
    col = torch.arange(table.shape[1], device=table.device)[None]
    full, part = kv_len[par] // page, (kv_len[par] % page != 0)
    off, ok, free = _plain_take(refs, part.long())
    own_page = free[off.clamp(max=P - 1)].int()
    last = part & ok
    src = torch.where(last, table[par, full.long().clamp(max=table.shape[1] - 1)], -1)
    dst = torch.where(last, own_page, -1)
    shared = torch.where((col < full[:, None]) & ok[:, None], table[par], -1)
    refs.scatter_add_(0, shared.clamp(min=0).reshape(-1).long(), (shared >= 0).int().reshape(-1))
    refs.scatter_add_(0, dst.clamp(min=0).long(), last.int())
    table[ch] = torch.where((col == full[:, None]) & last[:, None], dst[:, None], shared)
    n_pages[ch] = torch.where(ok, full + part.int(), 0).int()
    kv_len[ch] = torch.where(ok, kv_len[par], 0)
    status = torch.where(ok, 0, 4).int()
    frm, to = torch.where(src >= 0, src, P - 1).long(), torch.where(src >= 0, dst, P - 1).long()
    s["k"][to] = s["k"][frm]
    s["v"][to] = s["v"][frm]
    # room for N more rows everywhere
    want = ((kv_len + c["N"] + page - 1) // page).int()
    grow = (want - n_pages).clamp(min=0)
    off, ok, free = _plain_take(refs, grow.long())
    place = (col >= n_pages[:, None]) & (col < want[:, None]) & ok[:, None]
    fresh = free[(off[:, None] + col - n_pages[:, None]).clamp(0, P - 1)].int()
    table = torch.where(place, fresh, table)
    refs.scatter_add_(0, torch.where(place, fresh, 0).reshape(-1).long(), place.int().reshape(-1))
    n_pages = torch.where(ok, torch.maximum(want, n_pages), n_pages)
    room = torch.where(ok, 0, 4).int()
    # one row was kept: what lies behind it, and behind the window, goes back
    keep = kv_len + 1
    drop = (col >= ((keep + page - 1) // page)[:, None])
    if c["window"]:
        drop |= (col * page >= c["sinks"]) & ((col + 1) * page - 1 <= (keep - c["window"])[:, None])
    drop &= (col < n_pages[:, None]) & (table >= 0)
    refs.scatter_add_(0, torch.where(drop, table, 0).reshape(-1).long(), -drop.int().reshape(-1))
    table = torch.where(drop, -1, table)
    n_pages = torch.minimum(n_pages, ((keep + page - 1) // page).int())
    return {"refs": refs, "table": table, "n_pages": n_pages, "kv_len": kv_len, "src": src.int(), "dst": dst.int(),
            "status": status, "room": room, "k": s["k"], "v": s["v"]}


# --------------------------------------------------------------------------------- the package's
def _own(s):
    import paper_2311_08252_b200 as rest
    c = s["case"]
    if c["op"] == "attn":
        rest.rest_paged_attention(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["mask"], 1.0 / math.sqrt(c["D"]),
                                  window=c["window"], sinks=c["sinks"], n_nodes=s["n_nodes"], out=s["out"],
                                  lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "accept":
        n, nodes, out = rest.rest_accept_sampled(s["logits"], s["tokens"], s["parents"], s["n_nodes"], s["uniforms"],
                                                 s["temperature"], s["top_p"], c["max_depth"])
        return {"len": n, "nodes": nodes, "tokens": out}
    if c["op"] == "rows":
        rest.rest_paged_kv_write(s["k"], s["v"], s["table"], s["kv_len"], s["k_new"], s["v_new"],
                                 n_nodes=s["n_nodes"])
        rest.rest_paged_kv_commit(s["k"], s["v"], s["table"], s["kv_len"], s["accept_nodes"], s["accept_len"],
                                  c["N"], new_kv_len=s["new_kv_len"])
        return {"k": s["k"], "v": s["v"], "kv_len": s["new_kv_len"]}
    refs, table, n_pages, kv_len = s["refs"].clone(), s["table"].clone(), s["n_pages"].clone(), s["kv_len"].clone()
    src, dst, status = rest.rest_pages_fork(refs, table, n_pages, kv_len, s["parent"], s["child"], c["page"])
    rest.rest_pages_copy(s["k"], s["v"], src, dst)
    room = rest.rest_pages_reserve(refs, table, n_pages, kv_len + c["N"], c["page"])
    rest.rest_pages_release(refs, table, n_pages, kv_len + 1, c["page"], window=c["window"], sinks=c["sinks"])
    return {"refs": refs, "table": table, "n_pages": n_pages, "kv_len": kv_len, "src": src, "dst": dst,
            "status": status, "room": room, "k": s["k"], "v": s["v"]}


def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "accept": _plain_accept, "rows": _plain_rows, "fork": _plain_fork}[
        state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------ work
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "attn":
        B, N, H, Hkv, D, L = (case[k] for k in ("B", "N", "H", "Hkv", "D", "L"))
        if case["ragged"]:                                 # lengths and trees are even between half and whole
            L, N = 0.75 * L, 0.75 * N
        keys = (min(L, case["window"] + case["sinks"]) if case["window"] else L) + N
        return {"bytes": B * (Hkv * keys * 2 + H * N * 2) * D * size, "flops": 4.0 * B * H * N * keys * D}
    if case["op"] == "accept":
        # the root's row, and about two accepted nodes' rows
        rows = 1 + min(2.0, case["max_depth"], 0.75 * case["N"] / 2)
        return {"bytes": case["B"] * rows * case["V"] * size, "flops": case["B"] * rows * case["V"] * 4.0}
    row = case["Hkv"] * case["D"] * size * 2
    if case["op"] == "rows":
        return {"bytes": case["B"] * row * 2.0 * (0.75 * case["N"] + 3), "flops": 0}
    F = case["contexts"] * case["each"]
    cells = (case["contexts"] + F) * -(-(case["L"] + case["N"]) // case["page"])
    return {"bytes": F * row * 2.0 * case["page"] * (1 - 1.0 / case["page"]) + 8.0 * cells, "flops": 0}


# ----------------------------------------------------------------------------------------- exact
def _exact_attn(s):
    c = s["case"]
    N, H, Hkv, D, page = (c[k] for k in ("N", "H", "Hkv", "D", "page"))
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        L, n = int(s["kv_len"][b]), int(s["n_nodes"][b])
        prefix = torch.arange(L, device="cuda")
        where = torch.cat([prefix, L + torch.arange(n, device="cuda")])
        stands = torch.cat([prefix, L - 1 + s["depth"][b, :n]])       # position of each key in its sequence
        sees = torch.cat([torch.ones((n, L), dtype=torch.bool, device="cuda"), s["seen"][b, :n, :n]], 1)
        if c["window"]:
            mine = L - 1 + s["depth"][b, :n, None]
            sees &= (stands[None] < c["sinks"]) | (mine - stands[None] < c["window"])
            some = sees.any(0)
            where, sees = where[some], sees[:, some]
        pages, rows = s["table"][b].long()[where // page], where % page
        for h in range(Hkv):
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            q = s["q"][b, :n, heads].double().transpose(0, 1)         # [G,n,D]
            x = torch.einsum("gnd,kd->gnk", q, s["k"][pages, h, rows].double()) / math.sqrt(D)
            x = torch.where(sees[None], x, -math.inf)
            lse[b, heads, :n] = torch.logsumexp(x, -1)
            out[b, :n, heads] = torch.einsum("gnk,kd->gnd", torch.softmax(x, -1),
                                             s["v"][pages, h, rows].double()).transpose(0, 1)
    return {"out": out, "lse": lse}


def _exact_rows(s):
    c = s["case"]
    page = c["page"]
    got = []
    for pool, fresh in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        pool = pool.clone()
        for b in range(c["B"]):
            L, n, k = int(s["kv_len"][b]), int(s["n_nodes"][b]), int(s["accept_len"][b])
            rows = list(range(n))
            for a, i in enumerate(s["accept_nodes"][b, :k].tolist()):
                rows[a] = i                                           # slot a ends with the row of the a-th node
            at = L + torch.arange(n, device="cuda")
            pool[s["table"][b].long()[at // page], :, at % page] = fresh[b, rows]
        got.append(pool.double())
    return {"k": got[0], "v": got[1], "kv_len": None}


def _exact_fork(s):
    c = s["case"]
    page = c["page"]
    k, v = s["k"].double(), s["v"].double()
    free = [p for p, n in enumerate(s["refs"].tolist()) if n == 0]
    lens, table = s["kv_len"].tolist(), s["table"].tolist()
    for f in s["parent"].tolist():
        if lens[f] % page and free:
            a, z = table[f][lens[f] // page], free.pop(0)
            k[z], v[z] = s["k"][a].double(), s["v"][a].double()
    none = dict.fromkeys(("refs", "table", "n_pages", "kv_len", "src", "dst", "status", "room"))
    return {**none, "k": k, "v": v}


def exact(case, seed):
    """The floating outputs in 64 bits; the sampled acceptance gives whole numbers only."""
    if case["op"] == "accept":
        return None
    return {"attn": _exact_attn, "rows": _exact_rows, "fork": _exact_fork}[case["op"]](prepare(case, seed))
