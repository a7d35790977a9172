"""Plain 64-bit forms of the key/value cache's calls, one sequence and one head at
a time, and bounds on how far the kernels may be from them."""
import math

import numpy as np
import torch

from paper_2607_26566_gb300 import KVCache, Store, put_descs

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last place of 1.0
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # and below the smallest normal number
DEV = torch.device("cuda", 0)


def make_cache(kv_heads, dim, dtype, lens, page=65536, layers=1, seed=0, spare=3, more=0, fill=0xFF):
    """A cache whose sequences hold lens[s] tokens in scattered pages. Every byte of
    the pool is `fill` (0xFF: NaN in either type)."""
    from paper_2607_26566_gb300 import page_tokens
    T = page_tokens(page, kv_heads, dim, dtype, layers)
    n = sum(-(-(L + more) // T) for L in lens) + spare
    st = Store(torch.full((n * page,), fill, dtype=torch.uint8, device=DEV), page)
    s, ids = st.put_batch(put_descs(np.zeros(n, np.uint64), nbytes=np.full(n, page)))
    st.check(s)
    st.check(st.free(np.random.default_rng(seed).permutation(ids)))
    c = KVCache(st, kv_heads, dim, dtype, layers=layers, max_seqs=max(1, len(lens)), max_tokens=max(max(lens, default=1) + more, 1))
    c.reserve([L + more for L in lens])
    return c


def rows_of(c):
    """The pool as [pages, layers, 2, kv_heads, T, dim] (a view)."""
    shape = (c.layers, 2, c.kv_heads, c.page_tokens, c.head_dim)
    x = c.store.pool.view(c.dtype).view(-1, c.store.page_bytes // 2)
    return x[:, :math.prod(shape)].view(-1, *shape)


def write_rows(c, s, layer, key, val):
    """key, val [tokens, kv_heads, dim] as the first slots of sequence s."""
    T, pages, rows = c.page_tokens, c.pages(s), rows_of(c)
    for j in range(len(key)):
        rows[pages[j // T], layer, 0, :, j % T] = key[j]
        rows[pages[j // T], layer, 1, :, j % T] = val[j]


def read_rows(c, s, layer, n):
    """[2, tokens, kv_heads, dim]: the first n slots of sequence s."""
    pg = torch.tensor(c.pages(s), device=DEV, dtype=torch.long)
    x = rows_of(c)[pg, layer]                               # [pages, 2, kv_heads, T, dim]
    x = x.permute(1, 0, 3, 2, 4).reshape(2, -1, c.kv_heads, c.head_dim)
    return x[:, :n]


def turn64(x, w, eps, cos, sin, pos, interleaved):
    """x [tokens, heads, dim] in 64 bits: norm and rotation."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    if cos is None:
        return x
    y = x.clone()
    half = cos.shape[1]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[pos, i].double()[:, None], sin[pos, i].double()[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attend64(q, key, val, scale, softcap=0.0, slopes=None, window=0, spans=None, tree=None):
    """q [m, heads, dim] over key, val [L, kv_heads, dim]: out, lse, and sum of p|v|
    and the largest |score| for the bounds."""
    m, H, D = q.shape
    L, K = key.shape[0], key.shape[1]
    ctx = L - m
    pos = torch.arange(ctx, L)
    kpos = torch.arange(L)
    j = torch.arange(L)
    if tree is not None:
        bits = torch.tensor([[(int(w) >> b) & 1 for b in range(m)] for w in tree], dtype=torch.bool).view(m, m)
        depth = bits.sum(1) - 1
        pos = ctx + depth
        kpos = torch.cat([torch.arange(ctx), pos])
        see = torch.cat([torch.ones(m, ctx, dtype=torch.bool), bits], 1)
    elif spans is not None:
        see = (j >= spans[:, :1]) & (j < spans[:, 1:])
    else:
        see = j <= pos[:, None]
    if window:
        see = see & (kpos > pos[:, None] - window)
    out, lse = torch.zeros(m, H, D, dtype=torch.float64), torch.zeros(m, H, dtype=torch.float64)
    spread, big = torch.zeros_like(out), torch.zeros_like(lse)
    for h in range(H):
        x = q[:, h].double() @ key[:, h // (H // K)].double().T * scale
        big[:, h] = x.masked_fill(~see, 0).abs().amax(-1) if L else 0
        if softcap:
            x = softcap * torch.tanh(x / softcap)
        if slopes is not None:
            x = x - float(slopes[h]) * (pos[:, None] - kpos).abs()
        x = x.masked_fill(~see, -math.inf)
        lse[:, h] = torch.logsumexp(x, -1)
        p = torch.exp(x - torch.where(lse[:, h] == -math.inf, torch.zeros(()).double(), lse[:, h])[:, None])
        v = val[:, h // (H // K)].double()
        out[:, h], spread[:, h] = p @ v, p @ v.abs()
    return out, lse, spread, big


def near_attend(got, got_lse, want, lse, spread, big, dtype, what=""):
    """out: rounded once (UNIT of the value), from weights rounded to 16 bits (UNIT of
    each term); a score, in fp32 from exact products, is within 2^-20 of its largest
    magnitude and a few units of exp2, 1e-5 in all for scores below 8; lse likewise."""
    err = (got.double().cpu() - want).abs()
    slack = 1e-5 + 2.0 ** -20 * big[..., None]
    bound = UNIT[dtype] * want.abs() + (UNIT[dtype] + slack) * 1.01 * spread + TINY[dtype]
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert (err <= bound).all(), f"{what}: {float((err / bound).max()):.3f} of the bound"
    if got_lse is not None:
        g = got_lse.double().cpu()
        empty = lse == -math.inf
        assert torch.equal(g == -math.inf, empty), f"{what}: empty rows"
        e = (g - lse)[~empty].abs()
        assert (e <= (1e-5 + 2.0 ** -20 * big + 2.0 ** -22 * lse.abs())[~empty]).all(), f"{what}: lse off by {float(e.max()):.3g}"


def words(n, rng, branch=3):
    """Ancestor words of a random tree of n nodes."""
    w = []
    for i in range(n):
        up = w[int(rng.integers(max(0, (i - 1) // branch), i))] if i else 0
        w.append(up | 1 << i)
    return torch.tensor([x - (1 << 64) if x >> 63 else x for x in w], dtype=torch.int64)
