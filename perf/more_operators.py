"""Performance cases of the calls that keep a key/value cache bounded.

A text model beside the store (perf/operators.py has its cache: pages of [layers, 2, kv_heads, T,
head_dim] rows of 16 bits) may run for longer than the store has pages. The operators:

* ``sinks``  -- attention in a window that the first few tokens stay visible beside.
* ``weigh``  -- the attention that each cached token got from new queries, summed over them and over the
                heads that share a key, added to what it got before.
* ``select`` -- of each key head's slots those that stay: the first few, the last few, and the ones of
                most accumulated attention; their weights moved together.
* ``evict``  -- the rows of the slots that stay moved together, in their pages.

``run`` computes them in elementary torch operations in fp32, rounded once at the end, or, where
``own`` is set, by the calls of the package.
"""
import math
import random

import numpy as np
import torch

own = False

KiB = 1 << 10
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one user's next token in a talk far beyond its window: the smallest attention
        dict(name="sinks_token", kind="sinks", dtype="bf16", seqs=1, tokens=1, ctx=5000, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, window=1024, sinks=4, cap=0.0, bias=False),
        # a decoding step of 64 such users
        dict(name="sinks_step", kind="sinks", dtype="bf16", seqs=64, tokens=1, ctx=16000, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, window=2048, sinks=4, cap=0.0, bias=False),
        # a prompt of 8k tokens through a window
        dict(name="sinks_prompt", kind="sinks", dtype="fp16", seqs=1, tokens=8190, ctx=0, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=2048, window=1024, sinks=16, cap=0.0, bias=False),
        # one user's token, a short context
        dict(name="weigh_token", kind="weigh", dtype="bf16", seqs=1, tokens=1, ctx=700, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, window=0, sinks=0, cap=0.0, bias=False, spans=False, decay=1.0),
        # a decoding step of 64 users whose contexts are spread up to 16k tokens
        dict(name="weigh_step", kind="weigh", dtype="bf16", seqs=64, tokens=1, ctx=16000, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=64, window=0, sinks=0, cap=0.0, bias=False, spans=False, decay=1.0),
        # what the last 32 tokens of nine prompts look at, before a cache is cut; seven heads to a key
        dict(name="weigh_observe", kind="weigh", dtype="fp16", seqs=9, tokens=32, ctx=7000, heads=28, kv_heads=4, dim=128,
             layers=1, page_kib=256, window=0, sinks=0, cap=0.0, bias=False, spans=False, decay=0.0),
        # all of a prompt of 8k tokens: the most products
        dict(name="weigh_prompt", kind="weigh", dtype="bf16", seqs=1, tokens=8190, ctx=0, heads=32, kv_heads=8, dim=128,
             layers=1, page_kib=2048, window=0, sinks=0, cap=0.0, bias=False, spans=False, decay=1.0),
        # one user's cache, a little over its budget
        dict(name="select_token", kind="select", seqs=1, len=1100, kv_heads=8, keep=1024, sinks=4, recent=64, coarse=False),
        # 64 users' caches of up to 16k slots, to 4k each
        dict(name="select_step", kind="select", seqs=64, len=16000, kv_heads=8, keep=4096, sinks=4, recent=256,
             coarse=False),
        # one long document, weights of few values (many are alike)
        dict(name="select_long", kind="select", seqs=1, len=131000, kv_heads=8, keep=8192, sinks=16, recent=1024,
             coarse=True),
        # one user's cache, a little over its budget
        dict(name="evict_token", kind="evict", dtype="bf16", seqs=1, len=1100, kv_heads=8, dim=128, layers=1, page_kib=64,
             keep=1024, sinks=4, recent=64),
        # 64 users' caches of up to 16k slots, to 4k each: the most bytes
        dict(name="evict_step", kind="evict", dtype="bf16", seqs=64, len=16000, kv_heads=8, dim=128, layers=1, page_kib=64,
             keep=4096, sinks=4, recent=256),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case of the same ranges: each operator, its sizes spread over their logarithm."""
    kind = rng.choice(["sinks", "sinks", "weigh", "weigh", "weigh", "select", "select", "evict"])
    heads, kv_heads = rng.choice([(32, 8), (16, 16), (16, 2), (28, 4), (8, 1), (40, 8)])
    if kind in ("select", "evict"):
        c = dict(kind=kind, kv_heads=kv_heads, len=_log(rng, 1, 131000) if kind == "select" else _log(rng, 400, 16000))
        c.update(seqs=_log(rng, 1, max(1, min(64, (8_000_000 if kind == "select" else 1_000_000) // (c["len"] * kv_heads)))))
        share = rng.choice([0.06, 0.25, 0.5, 0.9, 1.1][:5 if kind == "select" else 4])  # (with 1.1 all of them stay)
        c.update(keep=max(1, int(c["len"] * share)), sinks=rng.choice([0, 4, 16]), recent=rng.choice([0, 64, 500]))
        if kind == "select":
            return dict(c, coarse=rng.random() < 0.4)
    else:
        c = dict(kind=kind, heads=heads, kv_heads=kv_heads)
    c.update(dtype=rng.choice(["bf16", "bf16", "fp16"]), dim=rng.choice([64, 80, 96, 128, 128]),
             layers=rng.choice([1, 1, 1, 2]), page_kib=rng.choice([64, 256, 2048]))
    while _page_tokens(c) < 8:
        c["page_kib"] *= 4
    if kind == "evict":
        return c
    c.update(cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.25, ctx=_log(rng, 1, 16000))
    if kind == "sinks":
        c.update(window=_log(rng, 8, 8000), sinks=_log(rng, 1, 256))
    else:
        c.update(window=rng.choice([0, 0, 0, _log(rng, 8, 8000)]), sinks=0, decay=rng.choice([0.0, 0.9, 1.0, 1.0]))
        if c["window"] and rng.random() < 0.5:
            c["sinks"] = _log(rng, 1, 256)
    c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
    rows = c["tokens"] * (c["ctx"] + c["tokens"])  # scores of one sequence and head
    c["seqs"] = _log(rng, 1, max(1, min(64, 26_000_000 // rows, 250_000 // (c["ctx"] + c["tokens"]))))
    if kind == "weigh":
        c["spans"] = c["tokens"] > 1 and rng.random() < 0.3
        if c["spans"]:
            c.update(window=0, sinks=0)
    return c


# ------------------------------------------------------------------ shapes
def _page_tokens(c):
    """Tokens of a page: the largest power of two whose rows fit."""
    n = c["page_kib"] * KiB // (c["layers"] * 4 * c["kv_heads"] * c["dim"])
    return 1 << (n.bit_length() - 1) if n else 0


def _sizes(c):
    """(new tokens, tokens in the cache with them) of each sequence; they belong to the case, not to the seed."""
    if "len" in c:
        r = random.Random(c["seqs"] * 1009 + c["len"])
        return [0] * c["seqs"], [c["len"]] + [r.randint(max(1, c["len"] // 4), c["len"]) for _ in range(c["seqs"] - 1)]
    r = random.Random(c["seqs"] * 1_000_003 + c["tokens"] * 1009 + c["ctx"])
    if c["tokens"] <= 32:
        new = [c["tokens"]] * c["seqs"]
    else:  # ragged around the mean, the first one as given
        new = [c["tokens"]] + [r.randint(max(1, c["tokens"] // 3), c["tokens"] * 5 // 3) for _ in range(c["seqs"] - 1)]
    ctx = [c["ctx"]] + [r.randint(c["ctx"] // 8, c["ctx"]) for _ in range(c["seqs"] - 1)]
    return new, [a + b for a, b in zip(new, ctx)]


def work(case):
    """Bytes read once and written once, and the products' operations on visible pairs."""
    c = case
    new, lens = _sizes(c)
    K = c["kv_heads"]
    if c["kind"] == "select":
        stay = sum(min(L, c["keep"]) for L in lens)
        return {"bytes": float(K * 4 * (sum(lens) + 2 * stay) + 8 * len(lens)), "flops": 0.0}
    row = 2 * c["dim"]
    if c["kind"] == "evict":  # (rows ahead of the first one that goes stay in place: the sinks, and a few)
        moved = sum(max(0, c["keep"] - c["sinks"]) for L in lens if L > c["keep"])
        return {"bytes": float(K * moved * (2 * 2 * row + 4)), "flops": 0.0}
    n, seen, pairs, got = sum(new), 0, 0, 0
    for k, (m, L) in enumerate(zip(new, lens)):
        first, last, head = _visible(c, k, m, L)
        head = np.minimum(head, first)
        pairs += int((np.maximum(last - first, 0) + head).sum())
        some = last > first
        mark = np.zeros(L + 1, np.int64)
        np.add.at(mark, first[some], 1)
        np.add.at(mark, last[some], -1)
        see = np.cumsum(mark)[:L] > 0
        see[:int(head.max())] = True
        seen += int(see.sum())
        if c["kind"] == "weigh":  # accumulated weights: read of old slots, written where they change
            ctx = L - m
            old = int(see[:ctx].sum()) if c["decay"] == 1.0 else ctx
            got += old * (8 if c["decay"] else 4) + 4 * m
    if c["kind"] == "weigh":
        return {"bytes": float(K * (seen * row + got) + n * c["heads"] * (row + 4)), "flops": 2.0 * pairs * c["heads"] * c["dim"]}
    return {"bytes": float(seen * 2 * K * row + 2 * n * c["heads"] * row + 4 * n * c["heads"]),
            "flops": 4.0 * pairs * c["heads"] * c["dim"]}


def _visible(c, k, m, L):
    """What each of sequence k's new tokens sees: slots [first, last), and the first `head`."""
    if c.get("spans"):
        first, last = _spans(c, k, m, L)
        return first, last, np.zeros(m, np.int64)
    p = np.arange(L - m, L)
    first = np.maximum(p - c["window"] + 1, 0) if c["window"] else np.zeros(m, np.int64)
    return first, p + 1, np.minimum(c["sinks"], p + 1)


def _spans(c, k, m, L):
    """Packed documents: a token sees its own document up to itself, the first document's tokens see all of
    it (a prefix), and the last token of the chunk is padding that sees nothing."""
    r = np.random.default_rng(k + m)
    cuts = np.unique(np.concatenate([[0], r.integers(0, L, 3)]))
    p = np.arange(L - m, L)
    doc = np.searchsorted(cuts, p, side="right") - 1
    ends = np.append(cuts[1:], L)
    first, last = cuts[doc], p + 1
    last = np.where(doc == 0, ends[0], last)
    first[-1] = last[-1] = 0
    return first, last


# ------------------------------------------------------------------ inputs
def _accumulated(c, lens, dev, g):
    """Weights [sequences, kv_heads, slots] as attention leaves them: most of it on few tokens, some tokens with none."""
    w = torch.randn(len(lens), c["kv_heads"], max(lens), device=dev, generator=g).mul_(2.0).exp_()
    w[torch.rand(w.shape, device=dev, generator=g) < 0.05] = 0.0
    if c.get("coarse"):
        w = (w * 16).floor_() / 16
    return w


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, lens = _sizes(c)
    K = c["kv_heads"]
    st = dict(c=c, max_new=max(new), max_len=max(lens), lens=torch.tensor(lens, dtype=torch.int32, device=dev),
              starts=torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=dev))
    if c["kind"] == "select":
        st.update(weights=_accumulated(c, lens, dev, g), **_kept(c, lens, dev))
        if own:
            from paper_2607_26566_gb300 import KVCache, Store
            st["store"] = Store(torch.empty(1 << 20, dtype=torch.uint8, device=dev), 1 << 20)
            st["cache"] = KVCache(st["store"], K, 64, max_seqs=len(lens), max_tokens=max(lens))
        return st
    dt, T, page = DTYPES[c["dtype"]], _page_tokens(c), c["page_kib"] * KiB
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
    st.update(T=T, pool=pool, table=torch.from_numpy(table).to(dev), layer=c["layers"] - 1)
    if own:
        from paper_2607_26566_gb300 import KVCache, Store, put_descs
        store = Store(pool, page)
        status, ids = store.put_batch(put_descs(np.zeros(n_pages, np.uint64), nbytes=np.full(n_pages, page)))
        store.check(status)
        store.check(store.free(ids[order]))
        cache = KVCache(store, K, c["dim"], dt, layers=c["layers"], max_seqs=len(lens), max_tokens=max(lens))
        cache.reserve(lens)
        st.update(store=store, cache=cache)
    if c["kind"] == "evict":
        chosen = dict(weights=_accumulated(c, lens, dev, g), lens=st["lens"], **_kept(c, lens, dev))
        _choose(chosen, c)
        st.update(kept=chosen["kept"], counts=chosen["counts"])
        return st
    n, H, D = sum(new), c["heads"], c["dim"]
    st["q"] = (2 * torch.randn(n, H, D, device=dev, generator=g)).to(dt)
    st["lse"] = torch.zeros(n, H, device=dev)
    st["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=dev) if c["bias"] else None
    if c.get("spans"):
        s = [np.stack(_spans(c, k, m, L), 1) for k, (m, L) in enumerate(zip(new, lens))]
        st["spans"] = torch.from_numpy(np.concatenate(s).astype(np.int32)).to(dev)
    if c["kind"] == "sinks":
        st["out"] = torch.zeros(n, H, D, dtype=dt, device=dev)
        return st
    # the sums that the attention before it left, and the weights so far
    x, _, tok, real = _scores(st, c)
    lse = torch.logsumexp(x, -1).permute(0, 3, 1, 2).flatten(2, 3)
    st["lse"][tok[real]] = lse[real]
    del x, lse
    st["weights"] = torch.rand(len(lens), K, max(lens) + 7, device=dev, generator=g)
    return st


def _kept(c, lens, dev):
    """Room for what is kept."""
    n, K = len(lens), c["kv_heads"]
    return dict(kept=torch.full((n, K, c["keep"]), -1, dtype=torch.int32, device=dev),
                counts=torch.zeros(n, dtype=torch.int32, device=dev), together=torch.zeros(n, K, c["keep"], device=dev))


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    return _own(s, c) if own else _plain(s, c)


def _own(s, c):
    cache = s["cache"]
    if c["kind"] == "select":
        cache.select(s["weights"], s["lens"], c["keep"], kept=s["kept"], counts=s["counts"], weights_out=s["together"],
                     recent=c["recent"], sinks=c["sinks"], max_len=s["max_len"])
        return {"kept": s["kept"], "counts": s["counts"], "weights": s["together"].view(torch.int32)}  # (moved: the same bits)
    if c["kind"] == "evict":
        cache.evict(s["kept"], s["counts"], layer=s["layer"])
        return {"pool": _rows(s, c).view(torch.int16)}  # moved, not computed: the same bits
    how = dict(starts=s["starts"], max_new=s["max_new"], layer=s["layer"], scale=c["dim"] ** -0.5, softcap=c["cap"],
               slopes=s["slopes"], window=c["window"], sinks=c["sinks"], max_len=s["max_len"])
    if c["kind"] == "weigh":
        cache.weigh(s["q"], s["lens"], s["lse"], s["weights"], spans=s.get("spans"), decay=c["decay"], **how)
        return {"weights": s["weights"]}
    cache.attend(s["q"], s["lens"], out=s["out"], lse=s["lse"], **how)
    return {"out": s["out"], "lse": s["lse"]}


def _rows(s, c):
    """The pool as [pages, layers, 2, kv_heads, T, dim]."""
    shape = (c["layers"], 2, c["kv_heads"], s["T"], c["dim"])
    x = s["pool"].view(DTYPES[c["dtype"]]).view(-1, c["page_kib"] * KiB // 2)
    return x[:, :math.prod(shape)].view(-1, *shape)


def _plain(s, c):
    if c["kind"] == "select":
        _choose(s, c)
        return {"kept": s["kept"], "counts": s["counts"], "weights": s["together"].view(torch.int32)}
    if c["kind"] == "evict":
        return _moved(s, c)
    x, see, tok, real = _scores(s, c)
    if c["kind"] == "weigh":
        lse = s["lse"][tok].view(*tok.shape, c["kv_heads"], -1).permute(0, 2, 3, 1)[..., None]
        w = torch.where((see & real[..., None])[:, None, None], torch.exp(x - lse), 0).sum((2, 3))
        lens, starts = s["lens"].long(), s["starts"].long()
        ctx = (lens - starts[1:] + starts[:-1])[:, None, None]
        j = torch.arange(s["max_len"], device=w.device)
        held = s["weights"][..., :s["max_len"]]
        w = torch.where(j < ctx, held * c["decay"], 0) + w
        held.copy_(torch.where(j < lens[:, None, None], w, held))
        return {"weights": s["weights"]}
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    p = p / torch.where(total == 0, 1, total)
    y = torch.matmul(p.flatten(2, 3), _cached(s, c, 1)).view(*x.shape[:-1], c["dim"])
    y, lse = y.permute(0, 3, 1, 2, 4).flatten(2, 3), lse.permute(0, 3, 1, 2).flatten(2, 3)
    s["out"][tok[real]] = y[real].to(s["out"].dtype)
    s["lse"][tok[real]] = lse[real]
    return {"out": s["out"], "lse": s["lse"]}


def _cached(s, c, which):
    """Keys or values of every sequence, padded: [sequences, kv_heads, slots, dim]."""
    x = _rows(s, c)[:, s["layer"], which][s["table"].long().clamp(min=0)].float()     # [B, pages, K, T, D]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[..., :s["max_len"], :]


def _scores(s, c):
    """Scores of every sequence at once, padded to the longest: [B, kv_heads, group, m, L], -inf where masked; which
    are seen [B, m, L]; the token of each row, and whether there is one."""
    dev, K, D = s["q"].device, c["kv_heads"], c["dim"]
    G, m, L = c["heads"] // K, s["max_new"], s["max_len"]
    lens, starts = s["lens"].long(), s["starts"].long()
    new = starts[1:] - starts[:-1]
    i = torch.arange(m, device=dev)
    real = i < new[:, None]                                               # [B, m]
    tok = torch.where(real, starts[:-1, None] + i, 0)
    q = s["q"].float()[tok].view(len(new), m, K, G, D)
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(len(new), K, G * m, D), _cached(s, c, 0).transpose(-1, -2))
    x = x.view(len(new), K, G, m, L) * D ** -0.5
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    j = torch.arange(L, device=dev)
    at = (lens - new)[:, None] + i                                        # positions of queries
    if s.get("spans") is not None:
        span = s["spans"].long()[tok]
        see = (j >= span[..., :1]) & (j < span[..., 1:])
    else:
        see = j <= at[..., None]
        if c["window"]:
            see = see & ((j > at[..., None] - c["window"]) | (j < c["sinks"]))
    if s["slopes"] is not None:
        far = (at[..., None] - j).abs().float()
        x = x - s["slopes"].view(K, G, 1, 1) * far[:, None, None]
    return torch.where(see[:, None, None], x, -math.inf), see, tok, real


def _choose(s, c):
    """kept, counts and the kept ones' weights of every sequence."""
    w, L = s["weights"], s["lens"].long()
    n = L.clamp(max=c["keep"])
    a = n.clamp(max=c["sinks"])
    b = torch.minimum(n - a, torch.full_like(n, c["recent"]))
    j = torch.arange(w.shape[2], device=w.device)
    # in the order in which they stay: sinks and recent ones, then by weight, then by slot; what is no slot last
    rank = torch.where((j < a[:, None]) | (j >= (L - b)[:, None]), 2, 1) * (j < L[:, None])
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(rank[:, None].expand_as(w).gather(-1, order), dim=-1, descending=True, stable=True).indices)
    place = torch.arange(w.shape[2], device=w.device) < n[:, None, None]
    stay = torch.zeros_like(w, dtype=torch.bool).scatter_(-1, order, place.expand_as(w))
    seq, head, slot = torch.nonzero(stay, as_tuple=True)
    to = (stay.cumsum(-1) - 1)[seq, head, slot]
    s["kept"][seq, head, to] = slot.int()
    s["together"][seq, head, to] = w[seq, head, slot]
    s["counts"].copy_(n)


def _moved(s, c):
    rows, T, table = _rows(s, c), s["T"], s["table"].long()
    seq, head, dst = torch.nonzero((torch.arange(s["kept"].shape[2], device=rows.device) < s["counts"][:, None, None])
                                   .expand_as(s["kept"]), as_tuple=True)
    src = s["kept"].long()[seq, head, dst]
    got = rows[table[seq, src // T], s["layer"], :, head, src % T]
    rows[table[seq, dst // T], s["layer"], :, head, dst % T] = got
    return {"pool": rows.view(torch.int16)}


# ------------------------------------------------------------------ from the definition, in 64 bits
def exact(case, seed):
    c = dict(case)
    if c["kind"] in ("select", "evict"):
        return None  # chosen and moved, nothing computed
    s = prepare(case, seed)
    new, lens = _sizes(c)
    T, dim, K, layer = s["T"], c["dim"], c["kv_heads"], s["layer"]
    table = s["table"].cpu().numpy()
    half_words = s["pool"].view(DTYPES[c["dtype"]])
    per_page = c["page_kib"] * KiB // 2
    e = torch.arange(dim, device="cuda")

    def row_of(k, slots, which):
        """[slots, kv_heads, dim] of sequence k in 64 bits."""
        page = table[k, slots // T].astype(np.int64) * per_page
        head = ((layer * 2 + which) * K + np.arange(K)) * T
        first = torch.from_numpy(page[:, None] + (head[None, :] + (slots % T)[:, None]) * dim).cuda()
        return half_words[first[..., None] + e].double()

    weigh = c["kind"] == "weigh"
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    held = s["weights"].double() if weigh else None
    G, at = c["heads"] // K, 0
    for k, (m, L) in enumerate(zip(new, lens)):
        key = row_of(k, np.arange(L), 0)
        val = None if weigh else row_of(k, np.arange(L), 1)
        first, last, head = (torch.from_numpy(np.asarray(b)).cuda()[:, None] for b in _visible(c, k, m, L))
        j = torch.arange(L, device="cuda")
        hidden = ~(((j >= first) | (j < head)) & (j < last))
        far = (torch.arange(L - m, L, device="cuda")[:, None] - j).abs().double()
        if weigh:
            held[k, :, :L - m] *= c["decay"]
            held[k, :, L - m:L] = 0
        for h in range(c["heads"]):
            step = max(1, (1 << 27) // L)
            for a in range(0, m, step):
                b = min(m, a + step)
                x = s["q"][at + a:at + b, h].double() @ key[:, h // G].T / math.sqrt(dim)
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if s["slopes"] is not None:
                    x = x - s["slopes"][h].double() * far[a:b]
                x = x.masked_fill(hidden[a:b], -math.inf)
                if weigh:
                    given = s["lse"][at + a:at + b, h].double()
                    held[k, h // G, :L] += torch.exp(x - torch.where(given == -math.inf, 0, given)[:, None]).sum(0)
                    continue
                l = torch.logsumexp(x, -1)
                lse[at + a:at + b, h] = l
                out[at + a:at + b, h] = torch.exp(x - torch.where(l == -math.inf, 0, l)[:, None]) @ val[:, h // G]
        at += m
    return {"weights": held} if weigh else {"out": out, "lse": lse}
