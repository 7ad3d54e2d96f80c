"""Rotary positions and the paged KV cache in 8 bits, as measurable cases.

    rotary   rest_rotary: queries (or keys) rotated by the positions of a draft's nodes
    append   rest_paged_kv_append, rest_paged_kv_append_scaled: a step's queries and keys rotated, keys and
             values written into 16-bit pages, or into e4m3 pages with a scale for 16 rows and head
    attn     rest_paged_attention_scaled: draft rows (or single tokens) over such a cache, with an
             optional sliding window and first tokens that stay visible
    commit   rest_paged_kv_commit_scaled, rest_pages_copy_scaled: the accepted path moved to the front, and the
             pages copied that a fork of the contexts needs

`own = False` computes them with elementary torch operations, `own = True` through the package."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
F8 = torch.float8_e4m3fn
BLOCK = 16                                                 # rows that share a scale


def listed():
    return [
        # the queries of one stream's draft tree, and of a batch whose heads are rotated in part, at far positions
        dict(name="rotary_b1", op="rotary", B=1, N=64, H=32, D=128, rot=128, pairs="half", far=4096, stretch=1.0,
             dtype="bf16"),
        dict(name="rotary_batch", op="rotary", B=128, N=64, H=32, D=128, rot=64, pairs="interleaved", far=1000000,
             stretch=8.0, dtype="fp16"),
        # one new token of one stream, and a draft tree's rows of a batch, into 8-bit pages
        dict(name="append_fp8_b1", op="append", B=1, N=1, H=32, Hkv=8, D=128, page=16, L=2048, rot=128, pairs="half",
             stretch=1.0, pages="fp8", dtype="bf16"),
        dict(name="append_fp8_batch", op="append", B=128, N=64, H=32, Hkv=8, D=128, page=64, L=1024, rot=128,
             pairs="half", stretch=1.0, pages="fp8", dtype="bf16"),
        # the same into 16-bit pages, ragged trees
        dict(name="append_16_batch", op="append", B=61, N=33, H=32, Hkv=8, D=128, page=16, L=4096, rot=128,
             pairs="interleaved", stretch=4.0, pages="16", dtype="bf16"),
        # one token of one stream: latency
        dict(name="attn_token_b1", op="attn", B=1, N=1, H=32, Hkv=8, D=128, page=16, L=2048, ragged=False, window=0,
             sinks=0, dtype="bf16"),
        # ordinary decoding of a large batch, uneven contexts
        dict(name="attn_tokens", op="attn", B=256, N=1, H=32, Hkv=8, D=128, page=64, L=4096, ragged=True, window=0,
             sinks=0, dtype="bf16"),
        # the same with small heads under a window
        dict(name="attn_tokens_window", op="attn", B=256, N=1, H=32, Hkv=8, D=64, page=128, L=8192, ragged=True,
             window=2048, sinks=64, dtype="fp16"),
        # a serving batch of draft trees, uneven prefixes and trees, grouped KV heads, small pages
        dict(name="attn_tree_batch", op="attn", B=61, N=64, H=32, Hkv=8, D=128, page=16, L=4096, ragged=True, window=0,
             sinks=0, dtype="bf16"),
        # large trees over long prefixes, five query heads per KV head
        dict(name="attn_tree_long", op="attn", B=16, N=128, H=40, Hkv=8, D=128, page=64, L=16384, ragged=False,
             window=0, sinks=0, dtype="bf16"),
        # the accepted path of one stream, and of a batch that is forked in two
        dict(name="commit_b1", op="commit", B=1, N=64, Hkv=8, D=128, page=16, L=2048, max_depth=10, fork=0),
        dict(name="commit_batch", op="commit", B=128, N=64, Hkv=32, D=128, page=64, L=1024, max_depth=16, fork=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "append", "attn", "attn", "attn", "commit"])
    dtype = rng.choice(["bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128, 256])
    D = rng.choice([64, 128])
    pairs, stretch = rng.choice(["half", "interleaved"]), rng.choice([1.0, 4.0, 8.0])
    if op == "rotary":
        D = rng.choice([64, 80, 96, 128, 256])
        N, H = _log(rng, 1, 256), rng.choice([1, 5, 8, 32, 40])
        return dict(op=op, B=_log(rng, 1, max(1, min(256, int(3.3e7 / (N * H * D))))), N=N, H=H, D=D,
                    rot=rng.choice([D, D // 2, 2 * rng.randint(1, D // 2)]), pairs=pairs, far=_log(rng, 10, 1000000),
                    stretch=stretch, dtype=rng.choice(["bf16", "fp16", "fp32"]))
    if op == "append":
        N, Hkv = rng.choice([1, _log(rng, 1, 256)]), rng.choice([1, 2, 4, 8, 32])
        H = Hkv * rng.choice([1, 3, 4, 5])
        return dict(op=op, B=_log(rng, 1, max(1, min(128, int(3.3e7 / (N * (H + 2 * Hkv) * D))))), N=N, H=H, Hkv=Hkv, D=D,
                    page=page, L=_log(rng, 1, 1024), rot=rng.choice([D, D // 2, 2 * rng.randint(1, D // 2)]), pairs=pairs,
                    stretch=stretch, pages=rng.choice(["fp8", "fp8", "16"]), dtype=dtype)
    if op == "attn":
        window = rng.choice([0, _log(rng, 40, 5000)])
        sinks = rng.choice([0, 4, rng.randint(1, 200)]) if window else 0
        Hkv, G, N = rng.choice([1, 2, 4, 8]), rng.choice([1, 3, 4, 5, 8]), rng.choice([1, 1, _log(rng, 1, 256)])
        L = _log(rng, 1, 16384)
        seen = (min(L, window + sinks) if window else L) + N
        most = min(256, int(2.5e8 / (Hkv * seen * D)), int(2.5e11 / (Hkv * G * N * seen * D * 4)),
                   int(1.3e9 / (Hkv * G * N * (L + N))), int(1e9 / (Hkv * (L + N) * D)))
        return dict(op=op, B=_log(rng, 1, max(1, most)), N=N, H=Hkv * G, Hkv=Hkv, D=D, page=page, L=L,
                    ragged=rng.random() < 0.7, window=window, sinks=sinks, dtype=dtype)
    B = _log(rng, 1, 128)
    return dict(op=op, B=B, N=_log(rng, 1, 256), Hkv=rng.choice([1, 4, 8, 32]), D=D, page=page, L=_log(rng, 1, 1024),
                max_depth=rng.randint(1, 16), fork=rng.choice([0, rng.randint(1, B)]))


# ---------------------------------------------------------------------------------------- inputs
def _trees(rng, B, N, max_depth, n_nodes):
    """Random trees: depth, ancestors [B,N,N], packed ancestor masks."""
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
    return depth, seen, words.view(np.int32).copy()


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


def _frequencies(rot, stretch):
    """One per pair, falling from 1 to nearly 1/10000; stretched for long contexts: pairs that turn once in more than
    1024 positions turn `stretch` times slower, those that turn faster than once in 128 as before, mixed between."""
    f = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    keep = np.clip((1024 * f / (2 * np.pi) - 1) / 7, 0, 1)
    return (f * (keep + (1 - keep) / stretch)).astype(np.float32), float(0.1 * math.log(stretch) + 1)


def prepare(case, seed):
    dev = torch.device("cuda")
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    to = lambda a, t=None: torch.from_numpy(np.ascontiguousarray(a)).to(dev, t)  # noqa: E731
    normal = lambda dt, *shape: torch.empty(shape, dtype=dt, device=dev).normal_(generator=gen)  # noqa: E731
    st = dict(case=dict(case))
    op, B, N, D = case["op"], case["B"], case["N"], case["D"]

    def cache(P):
        """Pages of codes that use their range, blocks of 16 rows at sizes of their own."""
        shape = (P, case["Hkv"], case["page"], D)
        for name in ("k", "v"):
            st[name] = torch.cat([normal(torch.float32, n, *shape[1:]).mul_(90.0).clamp_(-448, 448).to(F8)
                                  for n in [min(256, P - p) for p in range(0, P, 256)]])
            st[name + "s"] = torch.exp2(to(rng.integers(-8, -5, (P, case["Hkv"], case["page"] // BLOCK)), torch.float32))

    if op in ("rotary", "append"):
        f, amplitude = _frequencies(case["rot"], case["stretch"])
        st.update(inv_freq=to(f), amplitude=float(np.float32(amplitude)))
    if op == "rotary":
        dt = DTYPES[case["dtype"]]
        depth, seen, words = _trees(rng, B, N, 10, np.full(B, N))
        st.update(x=normal(dt, B, N, case["H"], D), out=torch.zeros((B, N, case["H"], D), dtype=dt, device=dev),
                  pos=to(rng.integers(0, case["far"], B)[:, None] + depth, torch.int32))
        return st
    lens = rng.integers((case["L"] + 1) // 2, case["L"] + 1, B) if case.get("ragged", op != "attn") else np.full(B, case["L"])
    nodes = rng.integers((N + 1) // 2, N + 1, B) if case.get("ragged", op != "attn") else np.full(B, N)
    depth, seen, words = _trees(rng, B, N, case.get("max_depth", 10), nodes)
    st.update(kv_len=to(lens, torch.int32), n_nodes=to(nodes, torch.int32))
    if op == "append":
        dt = DTYPES[case["dtype"]]
        table, P = _tables(rng, lens, N, case["L"] + N, case["page"], 0, 0, 1)
        if case["pages"] == "fp8":
            cache(P)
        else:
            st.update(k=normal(dt, P, case["Hkv"], case["page"], D), v=normal(dt, P, case["Hkv"], case["page"], D))
        # some tokens are louder than those before them
        loud = torch.exp2(to(rng.integers(0, 3, (B, N, 1, 1)), torch.float32))
        st.update(table=to(table), pos=to(lens[:, None] + depth - 1, torch.int32), q=normal(dt, B, N, case["H"], D),
                  q_out=torch.zeros((B, N, case["H"], D), dtype=dt, device=dev),
                  k_new=(normal(dt, B, N, case["Hkv"], D) * loud).to(dt), v_new=(normal(dt, B, N, case["Hkv"], D) * loud).to(dt))
    elif op == "attn":
        dt, H, L = DTYPES[case["dtype"]], case["H"], case["L"]
        window, sinks = case["window"], case["sinks"]
        table, P = _tables(rng, lens, N, min(L, window + sinks + 3 * case["page"] if window else L) + N, case["page"],
                           window, sinks, 1)
        cache(P)
        # some heads look at their keys more sharply than others
        sharp = torch.linspace(0.5, 2.0, H, device=dev)[None, None, :, None]
        st.update(q=(normal(dt, B, N, H, D).float() * sharp).to(dt), table=to(table), mask=to(words), depth=to(depth),
                  seen=to(seen), out=torch.zeros((B, N, H, D), dtype=dt, device=dev),
                  lse=torch.zeros((B, H, N), dtype=torch.float32, device=dev))
    else:
        table, P = _tables(rng, lens, N, case["L"] + N, case["page"], 0, 0, 1 + case["fork"])
        cache(P)
        # the accepted path: a random node's, from the root
        leaf = rng.integers(0, nodes)
        path = np.full((B, case["max_depth"]), -1, np.int32)
        on = seen[np.arange(B), leaf]
        rank = np.cumsum(on, 1) - 1
        bb, nn = np.nonzero(on)
        path[bb, rank[bb, nn]] = nn
        # a fork's copies: the last page of the first contexts into pages of their own
        ends = lens + on.sum(1) - 1
        src = table[np.arange(B), ends // case["page"]][:case["fork"]]
        st.update(table=to(table), accept_nodes=to(path), accept_len=to(on.sum(1), torch.int32),
                  new_kv_len=torch.zeros(B, dtype=torch.int32, device=dev), src=to(src, torch.int32),
                  dst=to(np.arange(P - 1 - case["fork"], P - 1), torch.int32))
    return st


# ------------------------------------------------------------------------------------ plain forms
def _turned(x, pos, inv_freq, amplitude, pairs):
    """x [B,N,H,D] in 64 bits, its first elements rotated: angles of far positions need the bits, and so do
    values next to the border between two codes."""
    half = inv_freq.shape[0]
    angle = pos.double()[:, :, None, None] * inv_freq.double()
    c, s = angle.cos() * amplitude, angle.sin() * amplitude
    x = x.double()
    head, tail = x[..., :2 * half], x[..., 2 * half:]
    if pairs == "half":
        x1, x2 = head[..., :half], head[..., half:]
        y = torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)
    else:
        x1, x2 = head[..., 0::2], head[..., 1::2]
        y = torch.stack([x1 * c - x2 * s, x2 * c + x1 * s], -1).flatten(-2)
    return torch.cat([y, tail], -1)


def _plain_rotary(s):
    return _turned(s["x"], s["pos"], s["inv_freq"], s["amplitude"], s["case"]["pairs"]).to(s["x"].dtype)


def _fitting(most):
    """The smallest power of two s with most <= 448 s (2^-60 at least)."""
    m, e = torch.frexp(most)
    return torch.exp2((torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-60).double()).masked_fill(most == 0, 2.0 ** -60)


def _plain_block_write(pool, scales, table, kv_len, n, fresh, page):
    """fresh [B,N,Hkv,D] in 64 bits, rows i < n[b] (n [B,1,1]), quantised into rows kv_len[b] + i, block by block."""
    B, N, Hkv, D = fresh.shape
    dev = pool.device
    b = torch.arange(B, device=dev)[:, None]
    L = kv_len.long()[:, None]
    blk = L // BLOCK + torch.arange(N // BLOCK + 2, device=dev)[None]                     # [B,J]
    i = (blk[:, :, None] * BLOCK + torch.arange(BLOCK, device=dev)) - L[:, :, None]       # [B,J,16]
    is_new = (i >= 0) & (i < n)
    kept = (i < 0) & is_new.any(2, keepdim=True)
    x = fresh[b[:, :, None], i.clamp(0, N - 1)]                                           # [B,J,16,Hkv,D]
    need = _fitting((x.abs() * is_new[..., None, None]).amax((2, 4)))                     # [B,J,Hkv]
    col = (blk * BLOCK // page).clamp(max=table.shape[1] - 1)
    live = is_new.any(2)
    pg = torch.where(live, table[b, col].long(), pool.shape[0] - 1)                       # others: the spare page
    cell, row = blk % (page // BLOCK), (blk * BLOCK) % page
    cell, row = torch.where(live, cell, 0), torch.where(live, row, 0)
    old = scales[pg, :, cell].double()                                                    # [B,J,Hkv]
    s = torch.where(kept.any(2)[..., None], torch.maximum(old, need), need)
    s = torch.where(live[..., None], s, old)
    at = row[:, :, None] + torch.arange(BLOCK, device=dev)                                # [B,J,16]
    was = pool[pg[:, :, None], :, at]                                                     # codes [B,J,16,Hkv,D]
    again = (was.double() * (old / s)[:, :, None, :, None]).to(F8)
    codes = (x / s[:, :, None, :, None]).to(F8)
    put = torch.where(is_new[..., None, None], codes.view(torch.uint8),
                      torch.where(kept[..., None, None], again.view(torch.uint8), was.view(torch.uint8)))
    pool.view(torch.uint8)[pg[:, :, None], :, at] = put
    scales[pg, :, cell] = s.float()


def _plain_append(s):
    c = s["case"]
    N, page = c["N"], c["page"]
    turn = lambda x: _turned(x, s["pos"], s["inv_freq"], s["amplitude"], c["pairs"])  # noqa: E731
    n = s["n_nodes"].long()[:, None, None]
    live = torch.arange(N, device=n.device)[None] < n[:, 0]
    out = {"q": torch.where(live[:, :, None, None], turn(s["q"]).to(s["q"].dtype), s["q_out"])}
    if c["pages"] == "fp8":
        _plain_block_write(s["k"], s["ks"], s["table"], s["kv_len"], n, turn(s["k_new"]), page)
        _plain_block_write(s["v"], s["vs"], s["table"], s["kv_len"], n, s["v_new"].double(), page)
        return {**out, "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}
    b = torch.arange(c["B"], device=n.device)[:, None]
    at = s["kv_len"].long()[:, None] + torch.arange(N, device=n.device)[None]
    pg, row = s["table"][b, (at // page).clamp(max=s["table"].shape[1] - 1)].long(), at % page
    for pool, fresh in ((s["k"], turn(s["k_new"]).to(s["k"].dtype)), (s["v"], s["v_new"])):
        pool[pg, :, row] = torch.where(live[:, :, None, None], fresh, pool[pg, :, row])
    return {**out, "k": s["k"], "v": s["v"]}


def _plain_attn(s):
    c = s["case"]
    B, N, H, Hkv, D, page = (c[k] for k in ("B", "N", "H", "Hkv", "D", "page"))
    G, W = H // Hkv, s["table"].shape[1]
    T = W * page
    rows = s["table"].clamp(min=0).long()

    def pages(codes, scales):
        x = codes.view(torch.uint8)[rows].view(F8).float().view(B, W, Hkv, page // BLOCK, BLOCK, D)
        x = x * scales[rows][..., None, None]
        return x.permute(0, 2, 1, 3, 4, 5).reshape(B, Hkv, T, D)

    k, v = pages(s["k"], s["ks"]), pages(s["v"], s["vs"])
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


def _plain_commit(s):
    c = s["case"]
    page, Hkv, D = c["page"], c["Hkv"], c["D"]
    b = torch.arange(c["B"], device=s["k"].device)[:, None]
    j = torch.arange(c["max_depth"], device=b.device)[None]
    moved = j < s["accept_len"][:, None]
    at = s["kv_len"].long()[:, None] + torch.where(moved, s["accept_nodes"].long(), 0)
    pg = s["table"][b, at // page].long()
    lens = s["accept_len"].long()[:, None, None]
    for pool, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        held = pool.view(torch.uint8)[pg, :, at % page].view(F8).double() * scales[pg, :, at % page // BLOCK].double()[..., None]
        _plain_block_write(pool, scales, s["table"], s["kv_len"], lens, held, page)
        src, dst = s["src"].long(), s["dst"].long()
        pool.view(torch.uint8)[dst] = pool.view(torch.uint8)[src]
        scales[dst] = scales[src]
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "kv_len": (s["kv_len"] + s["accept_len"]).int()}


# --------------------------------------------------------------------------------- the package's
def _own(s):
    import paper_2311_08252_b200 as rest
    c = s["case"]
    if c["op"] == "rotary":
        return rest.rest_rotary(s["x"], s["pos"], s["inv_freq"], interleaved=c["pairs"] == "interleaved",
                                amplitude=s["amplitude"], out=s["out"])
    if c["op"] == "append":
        turn = dict(positions=s["pos"], inv_freq=s["inv_freq"], interleaved=c["pairs"] == "interleaved",
                    amplitude=s["amplitude"], n_nodes=s["n_nodes"], q=s["q"], q_out=s["q_out"])
        if c["pages"] == "fp8":
            rest.rest_paged_kv_append_scaled(s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"], s["k_new"], s["v_new"],
                                          **turn)
            return {"q": s["q_out"], "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}
        rest.rest_paged_kv_append(s["k"], s["v"], s["table"], s["kv_len"], s["k_new"], s["v_new"], **turn)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if c["op"] == "attn":
        rest.rest_paged_attention_scaled(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"], s["mask"],
                                      1.0 / math.sqrt(c["D"]), window=c["window"], sinks=c["sinks"], n_nodes=s["n_nodes"],
                                      out=s["out"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    rest.rest_paged_kv_commit_scaled(s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"], s["accept_nodes"],
                                  s["accept_len"], c["N"], new_kv_len=s["new_kv_len"])
    if c["fork"]:
        rest.rest_pages_copy_scaled(s["k"], s["v"], s["ks"], s["vs"], s["src"], s["dst"])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "kv_len": s["new_kv_len"]}


def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attn": _plain_attn, "commit": _plain_commit}[
        state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------ work
def work(case):
    op, B, N, D = case["op"], case["B"], case["N"], case["D"]
    size = 4 if case.get("dtype") == "fp32" else 2
    if op == "rotary":
        return {"bytes": 2.0 * B * N * case["H"] * D * size, "flops": 3.0 * B * N * case["H"] * case["rot"]}
    Hkv = case["Hkv"]
    if op == "append":
        rows = B * (0.75 * N if N > 1 else 1)              # trees are even between half and whole
        to = 1 if case["pages"] == "fp8" else 2
        return {"bytes": rows * D * (case["H"] * 4.0 + 2 * Hkv * (2 + to)),
                "flops": 3.0 * rows * case["rot"] * (case["H"] + Hkv)}
    if op == "attn":
        H, L = case["H"], case["L"]
        if case["ragged"]:                                 # lengths and trees are even between half and whole
            L, N = 0.75 * L, (0.75 * N if N > 1 else 1)
        keys = (min(L, case["window"] + case["sinks"]) if case["window"] else L) + N
        return {"bytes": B * (Hkv * keys * 2 * (D + 4.0 / BLOCK) + H * N * 2 * D * size), "flops": 4.0 * B * H * N * keys * D}
    # about three rows move; a fork copies pages
    return {"bytes": 4.0 * Hkv * D * (3 * B + case["fork"] * case["page"]), "flops": 0}


# ----------------------------------------------------------------------------------------- exact
def _exact_turn(x, pos, s):
    """The rotation as a product of complex numbers."""
    f, half = s["inv_freq"].double(), s["inv_freq"].shape[0]
    angle = pos.double()[..., None] * f
    unit = torch.polar(torch.full_like(angle, s["amplitude"]), angle).unsqueeze(-2)
    x = x.double().clone()
    if s["case"]["pairs"] == "half":
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * unit
        x[..., :half], x[..., half:2 * half] = z.real, z.imag
    else:
        z = torch.complex(x[..., 0:2 * half:2].contiguous(), x[..., 1:2 * half:2].contiguous()) * unit
        x[..., 0:2 * half:2], x[..., 1:2 * half:2] = z.real, z.imag
    return x


def _exact_blocks(pool, scales, table, L, fresh, page):
    """fresh [n,Hkv,D] becomes rows L ... of one context (pool and scales change in place)."""
    n = fresh.shape[0]
    for first in range(L // BLOCK * BLOCK, L + n, BLOCK):
        lo, hi = max(first, L), min(first + BLOCK, L + n)
        p, cell, at = int(table[first // page]), first % page // BLOCK, first % page
        new = fresh[lo - L:hi - L]
        most = new.abs().amax((0, 2)) / 448
        s = torch.exp2(torch.ceil(torch.log2(most.clamp(min=2.0 ** -60))))
        s = torch.where(s / 2 >= most, s / 2, s).clamp(min=2.0 ** -60)       # (a logarithm a rounding too large)
        if lo > first:
            old = scales[p, :, cell].double()
            s = torch.maximum(s, old)
            kept = pool[p, :, at:at + lo - first].double() * (old / s)[:, None, None]
            pool[p, :, at:at + lo - first] = kept.to(F8)
        pool[p, :, at + lo - first:at + hi - first] = (new.transpose(0, 1) / s[:, None, None]).to(F8)
        scales[p, :, cell] = s.float()


def _exact_append(s):
    c = s["case"]
    q = s["q_out"].double()
    lens, nodes = s["kv_len"].tolist(), s["n_nodes"].tolist()
    k, v = _exact_turn(s["k_new"], s["pos"], s), s["v_new"].double()
    turned = _exact_turn(s["q"], s["pos"], s)
    table = s["table"].tolist()
    for b, (L, n) in enumerate(zip(lens, nodes)):
        q[b, :n] = turned[b, :n]
        if c["pages"] == "fp8":
            _exact_blocks(s["k"], s["ks"], table[b], L, k[b, :n], c["page"])
            _exact_blocks(s["v"], s["vs"], table[b], L, v[b, :n], c["page"])
    if c["pages"] == "fp8":
        return {"q": q, "k": s["k"].double(), "v": s["v"].double(), "ks": s["ks"].double(), "vs": s["vs"].double()}
    got = []
    for pool, fresh in ((s["k"].double(), k), (s["v"].double(), v)):
        for b, (L, n) in enumerate(zip(lens, nodes)):
            at = L + torch.arange(n, device="cuda")
            pool[s["table"][b].long()[at // c["page"]], :, at % c["page"]] = fresh[b, :n]
        got.append(pool)
    return {"q": q, "k": got[0], "v": got[1]}


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
        value = lambda codes, scales: (codes.view(torch.uint8)[pages, :, rows].view(F8).double() *  # noqa: E731
                                       scales[pages, :, rows // BLOCK].double()[..., None])
        k, v = value(s["k"], s["ks"]), value(s["v"], s["vs"])         # [keys,Hkv,D]
        for h in range(Hkv):
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            q = s["q"][b, :n, heads].double().transpose(0, 1)         # [G,n,D]
            x = torch.einsum("gnd,kd->gnk", q, k[:, h]) / math.sqrt(D)
            x = torch.where(sees[None], x, -math.inf)
            lse[b, heads, :n] = torch.logsumexp(x, -1)
            out[b, :n, heads] = torch.einsum("gnk,kd->gnd", torch.softmax(x, -1), v[:, h]).transpose(0, 1)
    return {"out": out, "lse": lse}


def _exact_commit(s):
    c = s["case"]
    page = c["page"]
    table, lens, paths = s["table"].tolist(), s["kv_len"].tolist(), s["accept_nodes"].tolist()
    for pool, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        for b, n in enumerate(s["accept_len"].tolist()):
            rows = [lens[b] + i for i in paths[b][:n]]
            held = torch.stack([pool[table[b][r // page], :, r % page].double() *
                                scales[table[b][r // page], :, r % page // BLOCK].double()[:, None] for r in rows])
            _exact_blocks(pool, scales, table[b], lens[b], held, page)
        for a, z in zip(s["src"].tolist(), s["dst"].tolist()):
            pool.view(torch.uint8)[z] = pool.view(torch.uint8)[a]
            scales[z] = scales[a]
    return {"k": s["k"].double(), "v": s["v"].double(), "ks": s["ks"].double(), "vs": s["vs"].double(), "kv_len": None}


def exact(case, seed):
    """The floating outputs in 64 bits (codes and scales: what the rounding of the exact values comes to)."""
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turn(s["x"], s["pos"], s)
    return {"append": _exact_append, "attn": _exact_attn, "commit": _exact_commit}[case["op"]](s)
