"""The key/value cache in the store's pages (marked gpu): each call against a plain
form in 64 bits, at the sizes, masks and places where it can go wrong. Every byte
of a pool that holds no row of the case is NaN."""
import math

import numpy as np
import pytest
import torch

from paper_2607_26566_gb300 import KVCache, Store, put_descs
from kv_plain import (DEV, TINY, UNIT, attend64, make_cache, near_attend, read_rows, rows_of, turn64, words, write_rows)

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def gen(seed):
    return torch.Generator().manual_seed(seed)


def starts_of(new):
    return torch.tensor(np.cumsum([0] + list(new)), dtype=torch.int32, device=DEV)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def tables(rows, half, seed=0):
    f = torch.exp(torch.arange(half).double() * (-math.log(10000.0) / max(1, half)))
    a = torch.arange(rows).double()[:, None] * f
    return a.cos().float().to(DEV), a.sin().float().to(DEV)


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,src", [(BF, BF), (HF, HF), (BF, FP), (HF, FP), (BF, HF), (HF, BF)])
@pytest.mark.parametrize("heads,kv,dim,rot,inter,norm", [
    (4, 2, 128, 128, False, True), (4, 2, 128, 128, True, False), (3, 1, 80, 80, False, True), (5, 5, 8, 8, True, True),
    (2, 1, 64, 40, False, False), (1, 1, 96, 96, True, True), (2, 2, 72, 2, False, True), (33, 3, 24, 0, False, True)])
def test_append(dtype, src, heads, kv, dim, rot, inter, norm):
    new, ctx, layers = [1, 0, 37, 64, 3], [15, 9, 0, 100, 62], 2
    lens = [a + b for a, b in zip(new, ctx)]
    c = make_cache(kv, dim, dtype, lens, layers=layers)
    before = rows_of(c).clone()
    n = sum(new)
    x = torch.randn(n, (heads + 2 * kv) * dim, generator=gen(dim)).to(src).to(DEV)      # a fused projection
    q, k, v = (y.view(n, -1, dim) for y in x.split([heads * dim, kv * dim, kv * dim], 1))
    w = (1 + 0.3 * torch.randn(2, dim, generator=gen(1))).to(DEV)
    cos, sin = tables(200, rot // 2) if rot else (None, None)
    out = torch.full((n, heads, dim), math.nan, dtype=dtype, device=DEV)
    c.append(k, v, ints(lens), q=q, q_out=out, starts=starts_of(new), max_new=64, layer=1, q_norm=w[0] if norm else None,
             k_norm=w[1] if norm else None, eps=1e-3, cos=cos, sin=sin, interleaved=inter)
    pos = torch.cat([torch.arange(L - m, L) for m, L in zip(new, lens)]).to(DEV)
    want_q = turn64(q, w[0] if norm else None, 1e-3, cos, sin, pos, inter)
    want_k = turn64(k, w[1] if norm else None, 1e-3, cos, sin, pos, inter)

    def close(got, want, name):
        # rounded once, from fp32: a few units in its last place of the head's largest element
        bound = UNIT[dtype] * 1.001 * want.abs() + 2.0 ** -20 * want.abs().amax(-1, keepdim=True) + TINY[dtype]
        assert ((got.double() - want).abs() <= bound).all(), name

    close(out, want_q, "q")
    at = 0
    for s, (m, L) in enumerate(zip(new, lens)):
        if m == 0:
            continue
        got = read_rows(c, s, 1, L)[:, L - m:]
        close(got[0], want_k[at:at + m], "k")
        assert torch.equal(got[1], v[at:at + m].to(dtype)), "v"
        at += m
    # nothing else was written
    after = rows_of(c).clone()
    for s, (m, L) in enumerate(zip(new, lens)):
        for j in range(L - m, L):
            pg = c.pages(s)[j // c.page_tokens]
            after[pg, 1, :, :, j % c.page_tokens] = before[pg, 1, :, :, j % c.page_tokens]
    assert torch.equal(after.view(torch.int16), before.view(torch.int16))


def test_append_in_place_positions_and_no_queries():
    c = make_cache(2, 64, BF, [5, 9])
    cos, sin = tables(40, 32)
    q, k, v = (torch.randn(4, h, 64, generator=gen(h)).to(BF).to(DEV) for h in (6, 2, 2))
    q0 = q.clone()
    pos = ints([39, 0, 7, 7])
    assert c.append(k, v, ints([5, 9]), q=q, q_out=q, cos=cos, sin=sin, positions=pos) is q   # two tokens each
    want = turn64(q0, None, 0, cos, sin, pos.long(), False)
    assert ((q.double() - want).abs() <= 2.0 ** -7.9 * want.abs() + 1e-5).all()
    got = read_rows(c, 1, 0, 9)[0, 7:]
    want = turn64(k, None, 0, cos, sin, pos.long(), False)[2:]
    assert ((got.double() - want).abs() <= 2.0 ** -7.9 * want.abs() + 1e-5).all()
    # keys and values only, and a position that the tables lack
    assert c.append(k, v, ints([5, 9]), cos=cos, sin=sin, positions=ints([40, -1, 0, 1])) is None
    got = read_rows(c, 0, 0, 5)[0, 3:]
    assert got.isnan().all()
    assert torch.equal(read_rows(c, 0, 0, 5)[1, 3:], v[:2])


def test_append_skips_what_has_no_place():
    c = make_cache(1, 64, HF, [8, 8])
    before = c.store.pool.clone()
    k = torch.zeros(4, 1, 64, dtype=HF, device=DEV)
    bad = ints([c.max_pages * c.page_tokens + 1, 1])       # past the table's end; more new tokens than tokens
    c.append(k, k, bad)
    c.append(k, k, ints([8, 8]), table=torch.full((2, 1), 1 << 30, dtype=torch.int32, device=DEV))  # no such page
    c.append(k, k, ints([8, 8]), table=torch.full((2, 1), -1, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before)


def test_append_of_many_sequences_finds_each_token_its_own():
    g = np.random.default_rng(4)
    new = g.integers(0, 4, 1500)
    ctx = g.integers(0, 20, 1500)
    lens = [int(a) for a in new + ctx]
    c = make_cache(1, 8, BF, lens, page=1024, more=1)
    n = int(new.sum())
    k = torch.arange(n, device=DEV, dtype=torch.float32).view(n, 1, 1).expand(n, 1, 8).contiguous()
    c.append(k, -k, ints(lens), starts=starts_of(new), max_new=3)
    at = 0
    rows = rows_of(c).cpu()
    for s in range(1500):
        for j in range(lens[s] - int(new[s]), lens[s]):
            r = rows[c.pages(s)[j // c.page_tokens], 0, :, 0, j % c.page_tokens, 0].float()
            want = torch.tensor([float(at), -float(at)]).to(BF).float()
            assert torch.equal(r, want), (s, j)
            at += 1
    assert at == n


# ------------------------------------------------------------------ attend
def case(dtype, heads, kv, dim, new, ctx, seed=0, page=65536, layers=1, qs=2.0):
    lens = [a + b for a, b in zip(new, ctx)]
    c = make_cache(kv, dim, dtype, lens, page=page, layers=layers, seed=seed)
    g = gen(seed)
    kvs = []
    for s, L in enumerate(lens):
        k, v = (torch.randn(L, kv, dim, generator=g).to(dtype) for _ in range(2))
        write_rows(c, s, layers - 1, k.to(DEV), v.to(DEV))
        kvs.append((k, v))
    q = (qs * torch.randn(sum(new), heads, dim, generator=g)).to(dtype)
    return c, lens, kvs, q


def check(c, lens, new, kvs, q, spans=None, tree=None, slopes=None, softcap=0.0, window=0, scale=None, max_len=0, each=False):
    n, heads, dim = q.shape
    out = torch.full((n, heads, dim), math.nan, dtype=c.dtype, device=DEV)
    lse = torch.full((n, heads), math.nan, device=DEV)
    how = dict(out=out, lse=lse, layer=c.layers - 1, softcap=softcap, window=window, scale=scale, max_len=max_len,
               slopes=None if slopes is None else slopes.to(DEV))
    if not each:
        how.update(starts=starts_of(new), max_new=max(new))
    for _ in range(2):  # the second call finds the workspace as the first one left it
        out.fill_(math.nan), lse.fill_(math.nan)
        if tree is not None:
            c.attend_tree(q.to(DEV), ints(lens), tree.to(DEV), **how)
        else:
            c.attend(q.to(DEV), ints(lens), spans=None if spans is None else spans.to(torch.int32).to(DEV), **how)
    at = 0
    for s, (m, L) in enumerate(zip(new, lens)):
        if m == 0:
            continue
        k, v = kvs[s]
        w = slice(at, at + m)
        want = attend64(q[w], k, v, dim ** -0.5 if scale is None else scale, softcap, slopes, window,
                        None if spans is None else spans[w], None if tree is None else tree[w])
        near_attend(out[w], lse[w], *want, c.dtype, f"sequence {s} of {m} new tokens, {L} in all")
        at += m
    return out, lse


HEADS = [(4, 4, 128), (8, 2, 128), (7, 1, 64), (6, 2, 80), (16, 1, 96), (2, 2, 8), (32, 2, 64)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_one_token(dtype, heads, kv, dim):
    new = [1] * 9
    ctx = [0, 1, 15, 16, 126, 127, 128, 700, 383]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    check(c, lens, new, kvs, q, each=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
@pytest.mark.parametrize("new,ctx", [([3, 0, 17, 1], [5, 40, 0, 300]), ([129, 64], [0, 200]), ([300], [77])])
def test_chunks(dtype, heads, kv, dim, new, ctx):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx, page=262144, layers=2)
    check(c, lens, new, kvs, q)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("queries", [16, 20, 32, 36, 64, 68])
def test_many_sequences_around_the_lines_between_kernels(dtype, heads, kv, dim, queries):
    """Hundreds of units, several to a block: at and past 16 and 32 queries to a
    key head, and past 64 row tiles; ragged, some sequences without a token."""
    most = queries * kv // heads
    new = [most if i % 3 == 0 else i % (most + 1) for i in range(330)]
    ctx = [(i * 37) % 300 for i in range(330)]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    check(c, lens, new, kvs, q)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("how", ["cap", "bias", "window", "all", "window1"])
@pytest.mark.parametrize("new,ctx", [([1, 1, 1], [0, 130, 700]), ([2, 9, 5], [3, 127, 400]), ([200, 40], [150, 0])])
def test_score_options(dtype, how, new, ctx):
    heads, kv, dim = 8, 2, 64
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx, qs=4.0)
    opt = {}
    if how in ("cap", "all"):
        opt["softcap"] = 5.0
    if how in ("bias", "all"):
        opt["slopes"] = torch.tensor([2.0 ** (-h - 1) for h in range(heads)])
    if how in ("window", "all"):
        opt["window"] = 100
    if how == "window1":
        opt["window"] = 1
    check(c, lens, new, kvs, q, scale=0.2, **opt)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 128), (3, 3, 80)])
@pytest.mark.parametrize("new,ctx", [([1, 1, 1, 1], [5, 200, 300, 0]), ([70, 0, 20], [0, 30, 260]), ([333], [5])])
@pytest.mark.parametrize("bias", [False, True])
def test_spans(dtype, heads, kv, dim, new, ctx, bias):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    g = np.random.default_rng(5)
    spans = []
    for m, L in zip(new, lens):
        for i in range(m):
            a, b = sorted(g.integers(0, L + 1, 2))
            pick = i % 4  # any span, none, all, one past its own slot (a later slot is visible)
            spans.append([(a, b), (b, a), (0, L), (max(0, L - m + i - 3), min(L, L - m + i + 2))][pick])
    slopes = torch.tensor([0.5 ** (h + 1) for h in range(heads)]) if bias else None
    out, lse = check(c, lens, new, kvs, q, spans=torch.tensor(spans), slopes=slopes)
    none = torch.tensor([b <= a for a, b in spans])
    assert none.any() or max(new) == 1
    assert (out.cpu()[none] == 0).all() and (lse.cpu()[none] == -math.inf).all()


def test_one_token_that_sees_nothing_beside_others():
    new, ctx = [1, 1, 1], [300, 0, 129]
    c, lens, kvs, q = case(HF, 4, 2, 64, new, ctx)
    out, lse = check(c, lens, new, kvs, q, spans=torch.tensor([[7, 7], [0, 1], [130, 2]]), each=True)
    assert (out[[0, 2]] == 0).all() and (lse[[0, 2]] == -math.inf).all()


def test_spans_beyond_the_sequence_are_cut():
    c, lens, kvs, q = case(BF, 2, 1, 64, [2, 1], [140, 3])
    spans = torch.tensor([[-5, 1 << 30], [141, 500], [2, 1 << 30]])
    how = torch.tensor([[0, 142], [141, 142], [2, 4]])
    out = torch.empty(3, 2, 64, dtype=BF, device=DEV)
    c.attend(q.to(DEV), ints(lens), out=out, starts=starts_of([2, 1]), max_new=2, spans=spans.to(torch.int32).to(DEV))
    a = attend64(q[:2], *kvs[0], 0.125, spans=how[:2])
    b = attend64(q[2:], *kvs[1], 0.125, spans=how[2:])
    near_attend(out[:2], None, *a, BF)
    near_attend(out[2:], None, *b, BF)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (4, 4, 64), (14, 2, 80), (64, 1, 128)])
@pytest.mark.parametrize("how", ["plain", "bias", "window"])
def test_tree(dtype, heads, kv, dim, how):
    rng = np.random.default_rng(dim)
    new = [1, 64, 21, 5]
    ctx = [30, 120, 0, 513]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    tree = torch.cat([words(m, rng) for m in new])
    opt = dict(slopes=torch.tensor([0.8 ** (h + 1) for h in range(heads)]), softcap=20.0) if how == "bias" else {}
    if how == "window":
        opt["window"] = 40
    check(c, lens, new, kvs, q, tree=tree, **opt)


def test_tree_words_that_see_nothing():
    c, lens, kvs, q = case(BF, 2, 1, 64, [3], [0])
    out = torch.full((3, 2, 64), math.nan, dtype=BF, device=DEV)
    lse = torch.zeros(3, 2, device=DEV)
    tree = torch.tensor([1, 0, 5], dtype=torch.int64)
    c.attend_tree(q.to(DEV), ints(lens), tree.to(DEV), out=out, lse=lse)
    want = attend64(q, *kvs[0], 0.125, tree=tree)
    near_attend(out, lse, *want, BF)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("heads,kv", [(4, 2), (2, 2)])
def test_many_short_sequences_beside_a_long_one(heads, kv):
    new = [300] + [2, 0, 1] * 25 + [129]
    ctx = [40] + [int(x) for x in np.random.default_rng(1).integers(0, 400, 75)] + [1]
    c, lens, kvs, q = case(BF, heads, kv, 64, new, ctx)
    check(c, lens, new, kvs, q)


@pytest.mark.parametrize("new", [[1, 1], [40, 3], [200, 30]])
@pytest.mark.parametrize("max_len", [1, 700, 1 << 30])
def test_a_wrong_max_len_changes_no_result(new, max_len):
    c, lens, kvs, q = case(HF, 4, 2, 64, new, [600, 90])
    check(c, lens, new, kvs, q, max_len=max_len)


def test_a_negative_scale_and_none():
    for new in ([1], [200]):
        c, lens, kvs, q = case(BF, 2, 1, 64, new, [300])
        check(c, lens, new, kvs, q, scale=-0.3)
        check(c, lens, new, kvs, q, scale=0.0)
        check(c, lens, new, kvs, q, scale=-0.2, softcap=3.0)


def test_starts_that_make_no_sense_touch_nothing():
    c, lens, kvs, q = case(BF, 2, 1, 64, [100, 100], [10, 10])
    out = torch.full((200, 2, 64), 7.0, dtype=BF, device=DEV)
    guard = torch.full((64,), 3.0, device=DEV)
    before = c.store.pool.clone()
    for starts in ([0, 200, 0], [500, 600, 700], [-50, -20, -10], [0, 1 << 30, 5]):
        c.attend(q.to(DEV), ints([5, 5]), out=out, starts=ints(starts), max_new=100)      # fewer slots than new tokens
        c.append(q[:, :1].contiguous().to(DEV), q[:, :1].contiguous().to(DEV), ints([5, 5]), starts=ints(starts), max_new=100)
    many = ints([0, 200] * 40)
    c2 = make_cache(1, 64, BF, [200] * 79, spare=0)
    c2.attend(q.to(DEV), ints([200] * 79), out=torch.empty_like(out), starts=many, max_new=200)  # more tokens than there are
    torch.cuda.synchronize()
    assert (out == 7).all() and (guard == 3).all() and torch.equal(c.store.pool, before)


def test_pages_beyond_4_gib():
    """A cache at the end of a 6 GiB pool: offsets pass 32 bits."""
    page = 1 << 20
    st = Store(torch.empty(6 << 30, dtype=torch.uint8, device=DEV), page)
    s, (filler,) = st.put_batch(put_descs([0], nbytes=[(6 << 30) - 4 * page]))
    st.check(s)
    c = KVCache(st, 2, 64, BF, max_seqs=2, max_tokens=3000)
    c.reserve([2500, 1200])
    assert min(c.pages(0) + c.pages(1)) >= 6 * 1024 - 4
    g = gen(3)
    q, k, v = (torch.randn(3700, h, 64, generator=g).to(BF) for h in (4, 2, 2))
    new = [2500, 1200]
    c.append(k.to(DEV), v.to(DEV), ints(new), starts=starts_of(new), max_new=2500)
    for s, w in ((0, slice(0, 2500)), (1, slice(2500, 3700))):
        assert torch.equal(read_rows(c, s, 0, new[s])[0].cpu(), k[w])
    pick = [2499, 3699]
    out = c.attend(q[pick].to(DEV), ints(new))
    near_attend(out[:1], None, *attend64(q[2499:2500], k[:2500], v[:2500], 0.125), BF)
    near_attend(out[1:], None, *attend64(q[3699:], k[2500:], v[2500:], 0.125), BF)
    whole = c.attend(q.to(DEV), ints(new), starts=starts_of(new), max_new=2500)
    near_attend(whole[2500:2600], None, *[x[:100] for x in attend64(q[2500:], k[2500:], v[2500:], 0.125)], BF)


def test_two_streams_and_a_graph():
    """Calls on two streams side by side have workspaces of their own; a graph of
    calls gives what the calls give."""
    c, lens, kvs, q = case(BF, 8, 2, 128, [1, 1, 1], [3000, 50, 1500])
    c2, lens2, kvs2, q2 = case(HF, 4, 1, 64, [150, 9], [700, 2000], seed=1)
    args, args2 = (q.to(DEV), ints(lens)), (q2.to(DEV), ints(lens2))
    how2 = dict(starts=starts_of([150, 9]), max_new=150)
    want, want2 = c.attend(*args), c2.attend(*args2, **how2)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got, got2 = [], []
    for _ in range(20):
        with torch.cuda.stream(a):
            got.append(c.attend(*args))
        with torch.cuda.stream(b):
            got.append(c.attend(*args))
            got2.append(c2.attend(*args2, **how2))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got) and all(torch.equal(x, want2) for x in got2)
    out, out2 = torch.zeros_like(want), torch.zeros_like(want2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(*args, out=out)
        c2.attend(*args2, out=out2, **how2)
    for _ in range(3):
        out.zero_(), out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want2)


@pytest.mark.parametrize("T", [8, 16, 128, 512])
def test_page_sizes(T):
    dim, kv = 64, 1
    page = T * 2 * kv * dim * 2
    new, ctx = [1, 40, 1, 2], [T * 3, T - 1, T * 2 - 1, 5]
    c, lens, kvs, q = case(BF, 4, kv, dim, new, ctx, page=page)
    assert c.page_tokens == T
    check(c, lens, new, kvs, q)


def test_rows_behind_a_window_may_hold_anything():
    c, lens, kvs, q = case(BF, 4, 2, 128, [1, 1], [700, 300])
    for s, L in enumerate(lens):  # NaN and infinities where no token looks
        k, v = kvs[s]
        k[:L - 50], v[:L - 50] = math.nan, math.inf
        write_rows(c, s, 0, k.to(DEV), v.to(DEV))
        k[:L - 50], v[:L - 50] = 0, 0
    check(c, lens, [1, 1], kvs, q, window=50)


def test_strides_and_a_table_of_chosen_rows():
    c, lens, kvs, q = case(HF, 6, 3, 64, [1, 1, 1, 1], [70, 10, 200, 33])
    pick = [2, 0]
    wide = torch.full((2, 20, 64), 7.0, dtype=HF, device=DEV)
    wide[:, 3:9] = q[pick].to(DEV)
    out = torch.full((2, 16, 64), 7.0, dtype=HF, device=DEV)
    table = torch.full((2, c.max_pages + 5), -1, dtype=torch.int32, device=DEV)
    table[:, 2:2 + c.max_pages] = c.table[pick]
    c.attend(wide[:, 3:9], ints([lens[i] for i in pick]), out=out[:, 4:10], table=table[:, 2:2 + c.max_pages])
    for r, i in enumerate(pick):
        near_attend(out[r:r + 1, 4:10], None, *attend64(q[i:i + 1], *kvs[i], 0.125), HF)
    assert (out[:, :4] == 7).all() and (out[:, 10:] == 7).all()


def test_pages_in_the_table_that_the_pool_lacks_read_as_zeros():
    c, lens, kvs, q = case(BF, 2, 1, 64, [1], [40])
    table = torch.full((1, c.max_pages), -1, dtype=torch.int32, device=DEV)
    out = c.attend(q.to(DEV), ints(lens), table=table)
    assert (out == 0).all()
    table.fill_(1 << 30)
    assert (c.attend(q.to(DEV), ints(lens), table=table) == 0).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rise", [3.0, 30.0, 200.0])
@pytest.mark.parametrize("new,ctx", [([1], [900]), ([20], [700]), ([300], [600])])
def test_scores_that_rise_from_tile_to_tile(dtype, rise, new, ctx):
    """Each 128 keys score `rise` above the ones before, some rows fall instead."""
    c, lens, kvs, q = case(dtype, 2, 1, 64, new, ctx, qs=1.0)
    k, v = kvs[0]
    k[:, :, :32] = (torch.arange(lens[0]) * (rise / 128 / 4)).to(dtype)[:, None, None] / 8
    q[:, :, :32] = 1.0
    q[::3, :, :32] = -1.0
    write_rows(c, 0, 0, k.to(DEV), v.to(DEV))
    check(c, lens, new, kvs, q, scale=1.0)


def test_infinite_scores_give_nan_like_the_formula():
    c, lens, kvs, q = case(BF, 1, 1, 64, [1], [20])
    q[:] = 1.0
    kvs[0][0][4] = math.inf
    write_rows(c, 0, 0, kvs[0][0].to(DEV), kvs[0][1].to(DEV))
    assert c.attend(q.to(DEV), ints(lens)).isnan().all()


# ------------------------------------------------------------------ commit
@pytest.mark.parametrize("dim,kv,layers,page", [(128, 2, 3, 65536), (8, 1, 1, 1024), (80, 3, 2, 65536)])
def test_commit(dim, kv, layers, page):
    ctx = [0, 7, 15, 30, 100]
    paths = [[0, 1, 2], [0, 3, 4, 9], [], [2, 3, 11, 12, 13, 14, 15, 16, 17, 40], [5]]
    most = 12
    c = make_cache(kv, dim, HF, [n + 64 for n in ctx], page=page, layers=layers, fill=0)
    c.store.pool.view(torch.int16).copy_(torch.randint(-30000, 30000, (c.store.pool.numel() // 2,), generator=gen(2), dtype=torch.int16))
    before = rows_of(c).view(torch.int16).clone()
    want = before.clone()
    T = c.page_tokens
    for s, p in enumerate(paths):
        pg = c.pages(s)
        for i, f in enumerate(p):
            a, b = ctx[s] + f, ctx[s] + i
            want[pg[b // T], :, :, :, b % T] = before[pg[a // T], :, :, :, a % T]
    path = torch.full((5, most), 63, dtype=torch.int32, device=DEV)
    for s, p in enumerate(paths):
        path[s, :len(p)] = ints(p)
    c.commit(ints(ctx), path, ints(len(p) for p in paths))
    assert torch.equal(rows_of(c).view(torch.int16), want)


def test_a_decoding_loop_follows_the_plain_one():
    """Prompt, steps, a drafted tree and its accepted path, through append, attend,
    attend_tree, commit and reserve, against attention over all accepted tokens."""
    heads, kv, dim = 8, 2, 64
    prompt = [50, 131]
    c = make_cache(kv, dim, BF, [1, 1], spare=60, more=399)
    g = gen(9)
    hist = [[], []]                          # accepted (k, v) of each sequence, as stored
    lens = [0, 0]

    def step(new, tree=None):
        n = sum(new)
        q, k, v = (torch.randn(n, h, dim, generator=g).to(BF) for h in (heads, kv, kv))
        now = [L + m for L, m in zip(lens, new)]
        qo = c.append(k.to(DEV), v.to(DEV), ints(now), q=q.to(DEV), starts=starts_of(new), max_new=max(new))
        lse = torch.empty(n, heads, device=DEV)
        how = dict(lse=lse, starts=starts_of(new), max_new=max(new), max_len=max(now))
        out = c.attend(qo, ints(now), **how) if tree is None else c.attend_tree(qo, ints(now), tree.to(DEV), **how)
        at = 0
        for s, m in enumerate(new):
            w = slice(at, at + m)
            kk = torch.cat([x for x, _ in hist[s]] + [k[w]])
            vv = torch.cat([x for _, x in hist[s]] + [v[w]])
            near_attend(out[w], lse[w], *attend64(q[w], kk, vv, dim ** -0.5, tree=None if tree is None else tree[w]), BF)
            at += m
        return k, v, now

    k, v, lens = step(prompt)
    hist = [[(k[:50], v[:50])], [(k[50:], v[50:])]]
    for _ in range(3):
        k, v, lens = step([1, 1])
        for s in range(2):
            hist[s].append((k[s:s + 1], v[s:s + 1]))
    rng = np.random.default_rng(0)
    for _ in range(2):
        tree = torch.cat([words(12, rng), words(12, rng)])
        k, v, now = step([12, 12], tree)
        paths = []
        for s in range(2):
            node = 11 - s
            paths.append([b for b in range(12) if int(tree[12 * s + node]) >> b & 1])
            keep = [12 * s + b for b in paths[s]]
            hist[s].append((k[keep], v[keep]))
        path = torch.zeros(2, 12, dtype=torch.int32, device=DEV)
        for s, p in enumerate(paths):
            path[s, :len(p)] = ints(p)
        c.commit(ints(lens), path, ints(len(p) for p in paths))
        lens = [L + len(p) for L, p in zip(lens, paths)]
    k, v, lens = step([2, 1])


# ------------------------------------------------------------------ pages and streams
def test_pages_follow_reserve_release_and_compaction():
    c = make_cache(1, 64, BF, [100, 300], page=4096, spare=30)
    st = c.store
    s, (dead,) = st.put_batch(put_descs([0], nbytes=[5 * st.page_bytes]))
    st.check(s)
    kvs = []
    for i, L in enumerate([100, 300]):
        k, v = (torch.randn(L, 1, 64, generator=gen(i)).to(BF) for _ in range(2))
        write_rows(c, i, 0, k.to(DEV), v.to(DEV))
        kvs.append((k, v))
    q = torch.randn(2, 2, 64, generator=gen(5)).to(BF)
    a = c.attend(q.to(DEV), ints([100, 300]))
    used = st.stats()["used_pages"]
    assert st.free([dead]) == 0
    s, moved = st.compact((used - 5) * st.page_bytes)
    st.check(s)
    c.refresh()
    assert all(p < used - 5 for i in range(2) for p in c.pages(i))
    assert torch.equal(c.attend(q.to(DEV), ints([100, 300])), a)
    c.release([0])
    assert c.pages(0) == [] and (c.table[0].cpu() == -1).all()
    assert st.stats()["used_pages"] == len(c.pages(1))
    c.close()
    assert st.stats()["used_pages"] == 0


def test_another_stream_waits_for_the_pages():
    """A put that reuses a sequence's pages, on another stream, waits for the appends
    and attentions that the cache's stream was given."""
    from paper_2607_26566_gb300 import get_descs, put_descs
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    c = make_cache(4, 128, BF, [1], spare=0, more=2047)
    c.hold(a)
    n = c._pages[0]
    k = torch.ones(2048, 4, 128, dtype=BF, device=DEV)
    q = torch.ones(1, 4, 128, dtype=BF, device=DEV)
    torch.cuda.synchronize()
    src = torch.full((n * c.store.page_bytes,), 0x55, dtype=torch.uint8, device=DEV)
    lens, one = ints([2048]), ints([2048])
    slow = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        for _ in range(20):
            slow = slow @ slow.clamp(-1e-3, 1e-3)
        c.append(k, k, lens)
        out = c.attend(q, one)
    c.release([0], stream=a)
    st, ids = c.store.put_batch(put_descs([src]), b)
    c.store.check(st)
    dst = torch.empty_like(src)
    st, _ = c.store.get_batch(get_descs(ids, [dst]), b)
    c.store.check(st)
    torch.cuda.synchronize()
    assert (out == 1).all()
    assert torch.equal(dst, src)


def test_a_full_store_refuses_and_changes_nothing():
    from paper_2607_26566_gb300 import T2IError
    c = make_cache(1, 64, BF, [10, 10], spare=1, more=5000)
    pages = [c.pages(0), c.pages(1)]
    with pytest.raises(ValueError):
        c.reserve([6000, 5000])
    c2 = type(c)(c.store, 1, 64, BF, max_seqs=2, max_tokens=50000)
    with pytest.raises(T2IError, match="NOSPACE"):
        c2.reserve([10, 50000])
    assert c2.pages(0) == [] and [c.pages(0), c.pages(1)] == pages


def test_a_failed_launch_is_reported():
    from paper_2607_26566_gb300 import T2IError
    c, lens, kvs, q = case(BF, 2, 1, 64, [1], [9])
    c.store.inject_launch_failure(1)
    with pytest.raises(T2IError, match="injected"):
        c.attend(q.to(DEV), ints(lens))
    check(c, lens, [1], kvs, q)


# ------------------------------------------------------------------ refusals
def test_refusals():
    from paper_2607_26566_gb300 import KVCache, T2IError
    c, lens, kvs, q = case(BF, 4, 2, 64, [2], [20])
    q, L = q.to(DEV), ints(lens)
    kv = torch.zeros(2, 2, 64, dtype=BF, device=DEV)
    cos, sin = tables(30, 32)
    ok = dict(q=q, q_out=torch.empty_like(q))
    before = c.store.pool.clone()
    wide = torch.zeros(2, 4 * 64 + 4, dtype=BF, device=DEV)
    overlapping = torch.zeros(3 * 4 * 64, dtype=BF, device=DEV)
    for why, call in {
        "table has no such layer": lambda: c.append(kv, kv, L, layer=1),
        "tokens do not divide": lambda: c.append(kv, kv, ints([22, 22, 22])[:3], table=c.table.expand(3, -1).contiguous()),
        "an output's rows overlap": lambda: c.append(kv, kv, L, q=q, q_out=overlapping.as_strided((2, 4, 64), (64, 64, 1))),
        "a stride of 260": lambda: c.attend(wide[:, :256].view(2, 4, 64), L),
        "an address off 16 bytes": lambda: c.attend(wide.view(-1)[4:516].view(2, 4, 64), L),
        "q_out on q's neighbour": lambda: c.append(kv, kv, L, q=overlapping[:512].view(2, 4, 64), q_out=overlapping[256:].view(2, 4, 64)),
        "out is q": lambda: c.attend(q, L, out=q),
        "heads": lambda: c.attend(q[:, :3].contiguous(), L),
        "a cap below 0": lambda: c.attend(q, L, softcap=-1.0),
        "scale": lambda: c.attend(q, L, scale=math.inf),
        "spans and a window": lambda: c.attend(q, L, spans=torch.zeros(2, 2, dtype=torch.int32, device=DEV), window=3),
        "starts without max_new": lambda: c.attend(q, L, starts=starts_of([2])),
        "a tree of 65": lambda: c.attend_tree(torch.zeros(65, 4, 64, dtype=BF, device=DEV), L, torch.zeros(65, dtype=torch.int64, device=DEV)),
        "eps": lambda: c.append(kv, kv, L, q_norm=torch.ones(64, device=DEV), eps=-1.0, **ok),
    }.items():
        with pytest.raises(T2IError, match="INVALID"):
            call()
            pytest.fail(why)
    for why, call in {
        "another dtype": lambda: c.attend(q.half(), L),
        "k and v differ": lambda: c.append(kv, kv.half(), L),
        "lens of 64 bits": lambda: c.attend(q, L.long()),
        "starts of 64 bits": lambda: c.attend(q, L, starts=starts_of([2]).long()),
        "positions": lambda: c.append(kv, kv, L, cos=cos, sin=sin, positions=torch.zeros(2, dtype=torch.int64, device=DEV)),
        "a norm's weights": lambda: c.append(kv, kv, L, k_norm=torch.ones(64, dtype=BF, device=DEV)),
        "a table": lambda: c.attend(q, L, table=c.table.long()),
        "a cache of fp32": lambda: KVCache(c.store, 1, 64, torch.float64),
    }.items():
        with pytest.raises(TypeError):
            call()
            pytest.fail(why)
    for why, call in {
        "heads apart": lambda: c.attend(q.transpose(0, 1).contiguous().transpose(0, 1), L),
        "lens for 2 sequences": lambda: c.attend(q, ints([22, 22])),
        "host lens": lambda: c.attend(q, L.cpu()),
        "cos without sin": lambda: c.append(kv, kv, L, cos=cos),
        "q_out alone": lambda: c.append(kv, kv, L, q_out=ok["q_out"]),
        "a shorter v": lambda: c.append(kv, kv[:1], L),
        "two dimensions": lambda: c.attend(q.view(2, -1), L),
        "lse of another shape": lambda: c.attend(q, L, lse=torch.zeros(2, 3, device=DEV)),
    }.items():
        with pytest.raises(ValueError):
            call()
            pytest.fail(why)
    for lay in (dict(kv_heads=1, head_dim=132), dict(kv_heads=1, head_dim=12), dict(kv_heads=0, head_dim=64),
                dict(kv_heads=1, head_dim=136), dict(kv_heads=64, head_dim=128), dict(kv_heads=1, head_dim=64, dtype=FP)):
        with pytest.raises(T2IError, match="INVALID"):
            KVCache(c.store, **lay)
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before)


def test_no_tokens_is_no_work():
    c = make_cache(1, 64, BF, [4])
    e = torch.empty(0, 1, 64, dtype=BF, device=DEV)
    launches = c.store.stats()["launches"]
    assert c.append(e, e, ints([4]), q=e).shape == (0, 1, 64)
    assert c.attend(e, ints([4])).shape == (0, 1, 64)
    c.commit(ints([]), torch.empty(0, 3, dtype=torch.int32, device=DEV), ints([]))
    assert c.store.stats()["launches"] == launches
