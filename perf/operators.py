"""Performance cases of the key/value cache in the store's pages.

A text model beside the store keeps its keys and values in pages of the same pool. A page holds
[layers, 2, kv_heads, T, head_dim] rows of 16 bits, T the largest power of two that fits; a
sequence's pages are listed in its row of an int32 table. The operators:

* ``append`` -- per-head RMS norm of new queries and keys and the rotation by position, keys and
                values written to their pages, queries to a buffer of their own.
* ``attend`` -- attention of new queries over the cache: one token a sequence to long chunks; scores
                capped by a tanh, a bias by distance, a window, or a span of visible keys for each
                query (document, prefix and padding masks).
* ``tree``   -- attention of a tree of drafted tokens, the last ones of each sequence: a query sees the
                context and its own ancestors.
* ``commit`` -- the rows of the accepted nodes of such trees moved together, in every layer.

``run`` computes them in elementary torch operations in fp32, rounded once at the end, or, where
``own`` is set, by the calls of the package.
"""
import math
import random

import numpy as np
import torch

own = False

KiB, MiB = 1 << 10, 1 << 20
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
POSITIONS = 1 << 15  # rows of the rotation's tables


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one user's next token: the smallest append, a fused projection's row to one page
        dict(name="append_token", kind="append", dtype="bf16", seqs=1, tokens=1, ctx=900, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, norm=False, rotary=128, interleaved=False, wide=False),
        # a decoding step of a full server, norms and the rotation, from fp32 projections
        dict(name="append_step", kind="append", dtype="bf16", seqs=192, tokens=1, ctx=800, heads=32, kv_heads=8,
             dim=128, layers=1, page_kib=64, norm=True, rotary=128, interleaved=False, wide=True),
        # ragged prompts of 8k tokens in all, rotation of interleaved pairs
        dict(name="append_prompts", kind="append", dtype="fp16", seqs=7, tokens=1200, ctx=0, heads=32, kv_heads=8,
             dim=128, layers=1, page_kib=256, norm=True, rotary=128, interleaved=True, wide=False),
        # one user, one token, a short context: the smallest attention
        dict(name="decode_token", kind="attend", dtype="bf16", seqs=1, tokens=1, ctx=700, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, cap=0.0, bias=False, window=0, spans=False),
        # a decoding step of 64 users whose contexts are spread up to 16k tokens
        dict(name="decode_step", kind="attend", dtype="bf16", seqs=64, tokens=1, ctx=16000, heads=32, kv_heads=8,
             dim=128, layers=1, page_kib=64, cap=0.0, bias=False, window=0, spans=False),
        # capped scores and a window, heads of 64, two layers to a page
        dict(name="decode_window", kind="attend", dtype="fp16", seqs=48, tokens=1, ctx=9000, heads=16, kv_heads=2,
             dim=64, layers=2, page_kib=256, cap=30.0, bias=False, window=4096, spans=False),
        # chunks of packed documents with a prefix each, a distance bias, heads of 80
        dict(name="chunk_documents", kind="attend", dtype="bf16", seqs=3, tokens=600, ctx=3000, heads=16, kv_heads=16,
             dim=80, layers=1, page_kib=64, cap=0.0, bias=True, window=0, spans=True),
        # a prompt of 8k tokens: the largest
        dict(name="prompt", kind="attend", dtype="bf16", seqs=1, tokens=8190, ctx=0, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=2048, cap=0.0, bias=False, window=0, spans=False),
        # one user's draft of 21 tokens
        dict(name="tree_draft", kind="tree", dtype="bf16", seqs=1, tokens=21, ctx=1500, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, cap=0.0, bias=False, window=0),
        # 24 users' drafts of 60 tokens, contexts up to 8k
        dict(name="tree_step", kind="tree", dtype="bf16", seqs=24, tokens=60, ctx=8000, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, cap=0.0, bias=False, window=0),
        # one user's accepted path, four layers to a page
        dict(name="commit_draft", kind="commit", dtype="bf16", seqs=1, tokens=21, ctx=1500, kv_heads=8, dim=128, layers=4,
             page_kib=256),
        # 96 users' accepted paths in 28 layers, 16 tokens to a 2 MiB page
        dict(name="commit_step", kind="commit", dtype="bf16", seqs=96, tokens=60, ctx=600, kv_heads=8, dim=128, layers=28,
             page_kib=2048),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case of the same ranges: each operator, its sizes spread over their logarithm."""
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "tree", "tree", "commit"])
    heads, kv_heads = rng.choice([(32, 8), (16, 16), (16, 2), (28, 4), (8, 1), (40, 8)])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16"]), heads=heads, kv_heads=kv_heads,
             dim=rng.choice([64, 80, 96, 128, 128]), layers=rng.choice([1, 1, 1, 2]), page_kib=rng.choice([64, 256, 2048]))
    while _page_tokens(c) < 8:
        c["page_kib"] *= 4
    if kind == "append":
        c.update(seqs=_log(rng, 1, 192), ctx=rng.choice([0, _log(rng, 1, 8000)]), norm=rng.random() < 0.5,
                 rotary=rng.choice([c["dim"], c["dim"], c["dim"] // 2, 0]), interleaved=rng.random() < 0.3,
                 wide=rng.random() < 0.2)
        c["tokens"] = _log(rng, 1, max(1, 8000 // c["seqs"]))
        return c
    if kind == "commit":
        c.update(seqs=_log(rng, 1, 96), tokens=rng.randint(8, 64), ctx=_log(rng, 1, 600), layers=rng.choice([1, 2, 4, 16]))
        del c["heads"]
        while _page_tokens(c) < 8:
            c["page_kib"] *= 4
        return c
    c.update(cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.25, window=rng.choice([0, 0, 0, _log(rng, 8, 8000)]))
    c["ctx"] = _log(rng, 1, 16000)
    if kind == "tree":
        c.update(tokens=rng.randint(1, 64))
        c["seqs"] = _log(rng, 1, max(1, min(48, 200_000 // (c["ctx"] + 64))))
        return c
    c["tokens"] = 1 if rng.random() < 0.5 else _log(rng, 2, 4096)
    rows = c["tokens"] * (c["ctx"] + c["tokens"])  # scores of one sequence and head
    c["seqs"] = _log(rng, 1, max(1, min(64, 40_000_000 // rows, 500_000 // (c["ctx"] + c["tokens"]))))
    c["spans"] = c["tokens"] > 1 and rng.random() < 0.3
    if c["spans"]:
        c["window"] = 0
    return c


# ------------------------------------------------------------------ shapes
def _page_tokens(c):
    """Tokens of a page: the largest power of two whose rows fit."""
    n = c["page_kib"] * KiB // (c["layers"] * 4 * c["kv_heads"] * c["dim"])
    return 1 << (n.bit_length() - 1) if n else 0


def _sizes(c):
    """(new tokens, tokens in the cache with them) of each sequence; they belong to the case, not to the seed."""
    r = random.Random(c["seqs"] * 1_000_003 + c["tokens"] * 1009 + c["ctx"])
    if c["kind"] in ("tree", "commit") or c["tokens"] == 1:
        new = [c["tokens"]] * c["seqs"]
    else:  # ragged around the mean, the first one as given
        new = [c["tokens"]] + [r.randint(max(1, c["tokens"] // 3), c["tokens"] * 5 // 3) for _ in range(c["seqs"] - 1)]
    ctx = [c["ctx"]] + [r.randint(c["ctx"] // 8, c["ctx"]) for _ in range(c["seqs"] - 1)]
    return new, [a + b for a, b in zip(new, ctx)]


def work(case):
    """Bytes read once and written once, and the products' operations on visible pairs."""
    c = case
    new, lens = _sizes(c)
    row = 2 * c["dim"]
    if c["kind"] == "commit":
        paths = _paths(c)
        moved = sum(int((p >= 0).sum()) - 1 for p in paths)  # the root stays where it is
        return {"bytes": float(moved * c["layers"] * 2 * c["kv_heads"] * row * 2), "flops": 0.0}
    n = sum(new)
    if c["kind"] == "append":
        src = 2 if c["wide"] else 1
        table = n * 8 * (c["rotary"] // 2)
        return {"bytes": float(n * row * (c["heads"] + 2 * c["kv_heads"]) * (1 + src) + table), "flops": 0.0}
    seen = pairs = 0
    for k, (m, L) in enumerate(zip(new, lens)):
        lo, hi = _visible(c, k, m, L)
        own_rows = 0
        if c["kind"] == "tree":
            t = _trees(c)[k]
            own_rows = int(sum(int(w).bit_count() for w in t))  # ancestors; a window over them counts as all
        pairs += int(np.maximum(hi - lo, 0).sum()) + own_rows
        some = hi > lo
        mark = np.zeros(L + 1, np.int64)
        np.add.at(mark, lo[some], 1)
        np.add.at(mark, hi[some], -1)
        seen += int((np.cumsum(mark) > 0).sum()) + (m if c["kind"] == "tree" else 0)
    return {"bytes": float(seen * 2 * c["kv_heads"] * row + 2 * n * c["heads"] * row),
            "flops": 4.0 * pairs * c["heads"] * c["dim"]}


def _visible(c, k, m, L):
    """Numpy bounds [lo, hi) of the cached slots that each of sequence k's new tokens sees (of a tree: of its context)."""
    p = np.arange(L - m, L)
    if c.get("spans"):
        return _spans(c, k, m, L)
    if c["kind"] == "tree":
        p = L - m + _depths(_trees(c)[k])
        hi = np.full(m, L - m)
    else:
        hi = p + 1
    lo = np.maximum(p - c["window"] + 1, 0) if c["window"] else np.zeros(m, np.int64)
    return np.minimum(lo, hi), hi


def _spans(c, k, m, L):
    """Packed documents: a token sees its own document up to itself, the first document's tokens see all of
    it (a prefix), and the last token of the chunk is padding that sees nothing."""
    r = np.random.default_rng(k + m)
    cuts = np.unique(np.concatenate([[0], r.integers(0, L, 3)]))
    p = np.arange(L - m, L)
    doc = np.searchsorted(cuts, p, side="right") - 1
    ends = np.append(cuts[1:], L)
    lo, hi = cuts[doc], p + 1
    hi = np.where(doc == 0, ends[0], hi)
    lo[-1] = hi[-1] = 0
    return lo, hi


def _trees(c):
    """Ancestor words [seqs, tokens]: bit j of word i is set where node i sees node j; a node sees itself."""
    r = random.Random(c["tokens"] * 31 + c["seqs"])
    out = np.zeros((c["seqs"], c["tokens"]), np.uint64)
    for s in range(c["seqs"]):
        for i in range(c["tokens"]):
            up = out[s, r.randint(max(0, (i - 1) // 3), max(0, i - 1))] if i else np.uint64(0)
            out[s, i] = up | (np.uint64(1) << np.uint64(i))
    return out


def _depths(words):
    return np.array([int(w).bit_count() - 1 for w in words], np.int64)


def _paths(c):
    """Accepted nodes of each tree, ascending, -1 after the last: the root, then nodes behind the path's own slots."""
    r = random.Random(c["tokens"] * 17 + c["seqs"])
    most = 8
    out = np.full((c["seqs"], most), -1, np.int64)
    for s in range(c["seqs"]):
        n = r.randint(1, min(most, c["tokens"] // 2) - 1)
        out[s, 0] = 0
        out[s, 1:n + 1] = sorted(r.sample(range(n + 1, c["tokens"]), n)) if n + 1 < c["tokens"] - n else range(n + 1, 2 * n + 1)
    return out


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = dict(case)
    dev, dt = torch.device("cuda"), DTYPES[c["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, lens = _sizes(c)
    T, page = _page_tokens(c), c["page_kib"] * KiB
    need = [-(-L // T) for L in lens]
    n_pages = sum(need) + 5
    pool = torch.empty(n_pages * page, dtype=torch.uint8, device=dev)
    pool.view(dt).normal_(generator=g)
    # a store in use: its free pages lie in any order. The last one freed is taken first
    order = np.random.default_rng(n_pages).permutation(n_pages)
    taken = order[::-1]
    table = np.full((len(lens), max(need)), -1, np.int32)
    at = 0
    for s, k in enumerate(need):
        table[s, :k] = taken[at:at + k]
        at += k
    st = dict(c=c, T=T, pool=pool, table=torch.from_numpy(table).to(dev), max_new=max(new), max_len=max(lens),
              lens=torch.tensor(lens, dtype=torch.int32, device=dev),
              starts=torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=dev))
    if own:
        from paper_2607_26566_gb300 import KVCache, Store, put_descs
        store = Store(pool, page)
        status, ids = store.put_batch(put_descs(np.zeros(n_pages, np.uint64), nbytes=np.full(n_pages, page)))
        store.check(status)
        store.check(store.free(ids[order]))
        cache = KVCache(store, c["kv_heads"], c["dim"], dt, layers=c["layers"], max_seqs=len(lens), max_tokens=max(lens))
        cache.reserve(lens)
        st.update(store=store, cache=cache)
    n, layer = sum(new), c["layers"] - 1
    st["layer"] = layer
    if c["kind"] == "commit":
        p = _paths(c)
        st.update(ctx=torch.tensor([L - c["tokens"] for L in lens], dtype=torch.int32, device=dev),
                  path=torch.from_numpy(p.astype(np.int32)).to(dev),
                  counts=torch.from_numpy((p >= 0).sum(1).astype(np.int32)).to(dev))
        return st
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    st["q_out"] = torch.zeros(n, H, D, dtype=dt, device=dev)
    if c["kind"] == "append":
        # one fused projection: queries, keys and values of a token in one row
        x = torch.randn(n, (H + 2 * K) * D, device=dev, generator=g)
        x = x if c["wide"] else x.to(dt)
        q, k, v = x.split([H * D, K * D, K * D], dim=1)
        st.update(q=q.view(n, H, D), k=k.view(n, K, D), v=v.view(n, K, D))
        if c["norm"]:
            st["wq"], st["wk"] = (1 + 0.2 * torch.randn(2, D, device=dev, generator=g)).unbind(0)
        if c["rotary"]:
            half = c["rotary"] // 2
            f = torch.exp(torch.arange(half, device=dev, dtype=torch.float64) * (-math.log(10000.0) / half))
            a = torch.arange(POSITIONS, device=dev, dtype=torch.float64)[:, None] * f
            st["cos"], st["sin"] = a.cos().float(), a.sin().float()
        return st
    st["q"] = (2 * torch.randn(n, H, D, device=dev, generator=g)).to(dt)
    st["lse"] = torch.zeros(n, H, device=dev)
    st["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=dev) if c["bias"] else None
    if c["kind"] == "tree":
        st["tree"] = torch.from_numpy(_trees(c).reshape(-1).view(np.int64)).to(dev)
    elif c["spans"]:
        s = [np.stack(_spans(c, k, m, L), 1) for k, (m, L) in enumerate(zip(new, lens))]
        st["spans"] = torch.from_numpy(np.concatenate(s).astype(np.int32)).to(dev)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    return _own(s, c) if own else _plain(s, c)


def _own(s, c):
    cache = s["cache"]
    if c["kind"] == "commit":
        cache.commit(s["ctx"], s["path"], s["counts"])
        return {"pool": _rows(s, c).view(torch.int16)}  # moved, not computed: the same bits
    ragged = dict(starts=s["starts"], max_new=s["max_new"])
    if c["kind"] == "append":
        cache.append(s["k"], s["v"], s["lens"], q=s["q"], q_out=s["q_out"], layer=s["layer"], q_norm=s.get("wq"),
                     k_norm=s.get("wk"), eps=EPS, cos=s.get("cos"), sin=s.get("sin"), interleaved=c["interleaved"], **ragged)
        return {"q": s["q_out"], "pool": _rows(s, c)}
    how = dict(out=s["q_out"], lse=s["lse"], layer=s["layer"], scale=c["dim"] ** -0.5, softcap=c["cap"], slopes=s["slopes"],
               window=c["window"], max_len=s["max_len"], **ragged)
    if c["kind"] == "tree":
        cache.attend_tree(s["q"], s["lens"], s["tree"], **how)
    else:
        cache.attend(s["q"], s["lens"], spans=s.get("spans"), **how)
    return {"out": s["q_out"], "lse": s["lse"]}


def _rows(s, c):
    """The pool as [pages, layers, 2, kv_heads, T, dim]."""
    shape = (c["layers"], 2, c["kv_heads"], s["T"], c["dim"])
    x = s["pool"].view(DTYPES[c["dtype"]]).view(-1, c["page_kib"] * KiB // 2)
    return x[:, :math.prod(shape)].view(-1, *shape)


def _owners(s):
    """(sequence, slot) of each new token."""
    n = int(s["q_out"].shape[0])
    i = torch.arange(n, device=s["pool"].device)
    seq = torch.searchsorted(s["starts"].long(), i, right=True) - 1
    return seq, s["lens"].long()[seq] - s["starts"].long()[seq + 1] + i


def _plain(s, c):
    rows = _rows(s, c)
    if c["kind"] == "commit":
        i = torch.arange(s["path"].shape[1], device=rows.device)
        seq, col = torch.nonzero(i < s["counts"][:, None], as_tuple=True)
        src = s["ctx"].long()[seq] + s["path"].long()[seq, col]
        dst = s["ctx"].long()[seq] + col
        table = s["table"].long()
        got = rows[table[seq, src // s["T"]], :, :, :, src % s["T"]]
        rows[table[seq, dst // s["T"]], :, :, :, dst % s["T"]] = got
        return {"pool": rows.view(torch.int16)}
    if c["kind"] == "append":
        seq, slot = _owners(s)
        q, k = _turned(s, c, s["q"].float(), s.get("wq"), slot), _turned(s, c, s["k"].float(), s.get("wk"), slot)
        page = s["table"].long()[seq, slot // s["T"]]
        rows[page, s["layer"], 0, :, slot % s["T"]] = k.to(rows.dtype)
        rows[page, s["layer"], 1, :, slot % s["T"]] = s["v"].to(rows.dtype)
        s["q_out"].copy_(q)
        return {"q": s["q_out"], "pool": rows}
    return _scores(s, c, rows)


def _turned(s, c, x, w, slot):
    """Norm over a head and rotation, in fp32."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    r = c["rotary"]
    if not r:
        return x
    cos, sin = s["cos"][slot][:, None], s["sin"][slot][:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
    return torch.cat([y, x[..., r:]], -1)


def _scores(s, c, rows):
    """Softmax attention of every sequence at once, padded to the longest."""
    dev, K, D = rows.device, c["kv_heads"], c["dim"]
    G, m, L = c["heads"] // K, s["max_new"], s["max_len"]
    kv = rows[:, s["layer"]][s["table"].long().clamp(min=0)].float()      # [B, pages, 2, K, T, D]
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, len(kv), K, -1, D)[..., :L, :]
    lens, starts = s["lens"].long(), s["starts"].long()
    new = starts[1:] - starts[:-1]
    i = torch.arange(m, device=dev)
    real = i < new[:, None]                                               # [B, m]
    tok = torch.where(real, starts[:-1, None] + i, 0)
    q = s["q"].float()[tok].view(len(new), m, K, G, D)
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(len(new), K, G * m, D), kv[0].transpose(-1, -2))
    x = x.view(len(new), K, G, m, L) * D ** -0.5
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    j = torch.arange(L, device=dev)
    ctx = (lens - new)[:, None]
    at, kpos = ctx + i, j.expand(len(new), L)                             # positions of queries and keys
    if c["kind"] == "tree":
        words = s["tree"][tok]                                            # [B, m]
        bits = (words[..., None] >> torch.arange(64, device=dev)) & 1
        depth = bits.sum(-1) - 1
        at = ctx + depth
        node = (j - ctx)                                                  # [B, L]
        drafted = (node >= 0) & (j < lens[:, None])
        node = node.clamp(0, m - 1)
        kpos = torch.where(drafted, ctx + depth.gather(1, node), kpos)
        see = torch.where(drafted[:, None], bits.gather(2, node[:, None].expand(-1, m, -1)) > 0, j < ctx[..., None])
    elif s.get("spans") is not None:
        span = s["spans"].long()[tok]
        see = (j >= span[..., :1]) & (j < span[..., 1:])
    else:
        see = j <= at[..., None]
    if c["window"]:
        see = see & (kpos[:, None] > at[..., None] - c["window"])
    if s["slopes"] is not None:
        far = (at[..., None] - kpos[:, None]).abs().float()
        x = x - s["slopes"].view(K, G, 1, 1) * far[:, None, None]
    x = torch.where(see[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    p = p / torch.where(total == 0, 1, total)
    y = torch.matmul(p.view(len(new), K, G * m, L), kv[1]).view(len(new), K, G, m, D)
    y, lse = y.permute(0, 3, 1, 2, 4).flatten(2, 3), lse.permute(0, 3, 1, 2).flatten(2, 3)
    s["q_out"][tok[real]] = y[real].to(s["q_out"].dtype)
    s["lse"][tok[real]] = lse[real]
    return {"out": s["q_out"], "lse": s["lse"]}


# ------------------------------------------------------------------ from the definition, in 64 bits
def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] == "commit":
        return None  # rows moved, nothing computed
    new, lens = _sizes(c)
    T, dim, K, layer = s["T"], c["dim"], c["kv_heads"], s["layer"]
    table = s["table"].cpu().numpy()
    half_words = s["pool"].view(DTYPES[c["dtype"]])
    per_page = c["page_kib"] * KiB // 2
    # element offset in the pool of the row of (sequence, slot, key or value, head)
    def offsets(k, slots, which):
        page = table[k, slots // T].astype(np.int64) * per_page
        head = ((layer * 2 + which) * K + np.arange(K)) * T
        return torch.from_numpy(page[:, None] + (head[None, :] + (slots % T)[:, None]) * dim).cuda()

    e = torch.arange(dim, device="cuda")
    if c["kind"] == "append":
        pool = half_words.double()
        q_out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for k, (m, L) in enumerate(zip(new, lens)):
            slots = np.arange(L - m, L)
            where = slice(at, at + m)
            q_out[where] = _turned64(s, c, s["q"][where].double(), s.get("wq"), slots)
            pool[offsets(k, slots, 0)[..., None] + e] = _turned64(s, c, s["k"][where].double(), s.get("wk"), slots)
            pool[offsets(k, slots, 1)[..., None] + e] = s["v"][where].double()
            at += m
        shape = (c["layers"], 2, K, T, dim)
        return {"q": q_out, "pool": pool.view(-1, per_page)[:, :math.prod(shape)].reshape(-1, *shape)}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    G, at = c["heads"] // K, 0
    trees = _trees(c) if c["kind"] == "tree" else None
    for k, (m, L) in enumerate(zip(new, lens)):
        slots = np.arange(L)
        key = half_words[offsets(k, slots, 0)[..., None] + e].double()       # [L, K, dim]
        val = half_words[offsets(k, slots, 1)[..., None] + e].double()
        lo, hi = (torch.from_numpy(np.asarray(b)).cuda()[:, None] for b in _visible(c, k, m, L))
        j = torch.arange(L, device="cuda")
        see = (j >= lo) & (j < hi)
        pos, kpos = torch.arange(L - m, L, device="cuda"), j.clone()
        if trees is not None:
            d = torch.from_numpy(_depths(trees[k])).cuda()
            pos = L - m + d
            kpos[L - m:] = pos
            up = np.array([[(int(w) >> b) & 1 for b in range(m)] for w in trees[k]], bool)
            see[:, L - m:] = torch.from_numpy(up).cuda()
            if c["window"]:
                see &= kpos > pos[:, None] - c["window"]
        far = (pos[:, None] - kpos).abs().double()
        for h in range(c["heads"]):
            step = max(1, (1 << 27) // L)
            for a in range(0, m, step):
                b = min(m, a + step)
                x = s["q"][at + a:at + b, h].double() @ key[:, h // G].T / math.sqrt(dim)
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if s["slopes"] is not None:
                    x = x - s["slopes"][h].double() * far[a:b]
                x = x.masked_fill(~see[a:b], -math.inf)
                l = torch.logsumexp(x, -1)
                lse[at + a:at + b, h] = l
                w = torch.exp(x - torch.where(l == -math.inf, 0, l)[:, None])
                out[at + a:at + b, h] = w @ val[:, h // G]
        at += m
    return {"out": out, "lse": lse}


def _turned64(s, c, x, w, slots):
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
    y = x.clone()
    t = torch.from_numpy(slots).cuda()
    for i in range(c["rotary"] // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rotary"] // 2)
        co, si = s["cos"][t, i].double()[:, None], s["sin"][t, i].double()[:, None]
        y[..., a], y[..., b] = x[..., a] * co - x[..., b] * si, x[..., b] * co + x[..., a] * si
    return y
