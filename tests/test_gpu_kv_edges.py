"""The key/value cache's scores and masks where they are hardest (marked gpu): short
drafts and chunks with every mask, weights far below the largest, large caps, far
positions, words with more bits than there are tokens."""
import math

import numpy as np
import pytest
import torch

from kv_plain import DEV, UNIT, attend64, make_cache, near_attend, words
from test_gpu_kv import BF, HF, case, check, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


# (heads, kv_heads, dim, most new tokens): 5 to 16 and 17 to 32 queries to a key head
FEW = [(2, 2, 64, 8), (4, 2, 80, 8), (8, 2, 128, 8), (5, 1, 64, 5), (4, 4, 128, 24), (2, 1, 96, 16)]


def options(how, heads):
    o = {}
    if how in ("window", "all"):
        o["window"] = 40
    if how in ("bias", "all"):
        o["slopes"] = torch.tensor([0.8 ** (h + 1) for h in range(heads)])
    if how in ("cap", "all"):
        o["softcap"] = 5.0
    return o


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim,most", FEW)
@pytest.mark.parametrize("how", ["plain", "window", "bias", "cap", "all"])
def test_short_drafts(dtype, heads, kv, dim, most, how):
    """Trees of few queries to a key head: contexts of none, in one tile, across the
    edge of a tile, and over several runs of tiles."""
    rng = np.random.default_rng(dim + most)
    new = [1, min(5, most), most, 3, 2]
    ctx = [0, 125, 700, 30, 2600]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    tree = torch.cat([words(m, rng) for m in new])
    check(c, lens, new, kvs, q, tree=tree, **options(how, heads))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim,most", FEW)
@pytest.mark.parametrize("how", ["plain", "bias", "cap"])
def test_spans_of_few_tokens(dtype, heads, kv, dim, most, how):
    """Spans that are any, empty, whole or look ahead, in one unit."""
    g = np.random.default_rng(dim + most)
    new = [1, min(5, most), most, 3, 2, 4]
    ctx = [0, 125, 700, 30, 2600, 0]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    spans = []
    for s, (m, L) in enumerate(zip(new, lens)):
        for i in range(m):
            a, b = sorted(int(x) for x in g.integers(0, L + 1, 2))
            spans.append([(a, b), (b, a), (0, L), (max(0, L - m + i - 3), min(L, L - m + i + 2))][(i + s) % 4])
    out, lse = check(c, lens, new, kvs, q, spans=torch.tensor(spans), **options(how, heads))
    none = torch.tensor([b <= a for a, b in spans])
    assert none.any() and not none.all()
    assert (out.cpu()[none] == 0).all() and (lse.cpu()[none] == -math.inf).all()


def one_strong_key(dtype, new, seqs, above, where):
    """`new` tokens of each of `seqs` sequences (on one sequence's pages) over 131,072
    keys of score 0, value 1, and one of score `above`, value 0; out and lse, each with
    what it should be and the bounds of near_attend."""
    n, L = 1 << 17, (1 << 17) + new
    c = make_cache(1, 64, dtype, [L], page=1 << 20)
    key, val = torch.zeros(L, 1, 64, dtype=dtype), torch.ones(L, 1, 64, dtype=dtype)
    key[where, 0, 0], val[where] = above, 0
    q = torch.zeros(new, 1, 64, dtype=dtype)
    q[:, 0, 0] = 1
    c.append(key.to(DEV), val.to(DEV), ints([L]))
    lse = torch.empty(new * seqs, 1, device=DEV)
    table = c.table[:1].expand(seqs, -1).contiguous()
    out = c.attend(q.to(DEV).repeat(seqs, 1, 1), ints([L] * seqs), lse=lse, scale=1.0, table=table)
    want, want_lse, spread, big = attend64(q, key, val, 1.0)
    slack = 1e-5 + 2.0 ** -20 * above
    bound = UNIT[dtype] * want + (UNIT[dtype] + slack) * 1.01 * spread
    return (out.double().cpu().view(seqs, new, 1, 64), want, bound,
            lse.double().cpu().view(seqs, new, 1), want_lse, slack + 2.0 ** -22 * want_lse.abs())


@pytest.mark.parametrize("new,seqs", [(1, 320), (24, 320), (40, 160)])
@pytest.mark.parametrize("above", [16.0, 17.0])
@pytest.mark.parametrize("where", [0, 131_071])
def test_sums_of_long_runs(new, seqs, above, where):
    """Over a run of a thousand tiles a sum keeps weights that are below half a unit of
    it one by one, and are 4e-5 to 1e-4 of it together."""
    out, want, bound, lse, want_lse, lse_bound = one_strong_key(BF, new, seqs, above, where)
    assert ((out - want).abs() <= bound).all()
    off = (lse - want_lse).abs()
    assert (off <= lse_bound).all(), f"{float(off.max()):.3g}"


@pytest.mark.parametrize("new,seqs", [(1, 320), (40, 160)])
@pytest.mark.parametrize("above", [17.0625, 18.0, 20.0])
@pytest.mark.parametrize("where", [0, 70_000, 131_071])
def test_many_keys_far_below_the_largest(new, seqs, above, where):
    """fp16: weights of 2^-24.6 to 2^-28.9 of the strong key's are all that the output
    consists of. A weight is off by 2^-32 of the largest at most."""
    out, want, bound, lse, want_lse, lse_bound = one_strong_key(HF, new, seqs, above, where)
    err = (out - want).abs()
    assert (err <= bound + 2.0 ** -32 * (1 << 17)).all(), f"{float((err / want).max()):.3f} of the output"
    assert ((lse - want_lse).abs() <= lse_bound).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("softcap", [1.0, 50.0, 1e3, 1e5, 1e7])
@pytest.mark.parametrize("new,ctx", [([1, 1], [300, 20]), ([5], [200]), ([70], [150])])
def test_caps_from_small_to_far_above_the_scores(dtype, softcap, new, ctx):
    c, lens, kvs, q = case(dtype, 4, 2, 64, new, ctx)
    check(c, lens, new, kvs, q, softcap=softcap)


@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("tree", [False, True])
def test_positions_that_fp32_cannot_count(new, tree):
    """Distances count exactly where positions are above 2^24 (and odd)."""
    ctx, window = (1 << 24) + 1001, 64
    L = ctx + new
    c = make_cache(1, 8, BF, [L], page=1 << 20)
    g = torch.Generator().manual_seed(new)
    key, val = (torch.randn(window + new, 1, 8, generator=g).to(BF) for _ in range(2))
    q = torch.randn(new, 1, 8, generator=g).to(BF)
    c.append(key.to(DEV), val.to(DEV), ints([L]))
    lse = torch.empty(new, 1, device=DEV)
    how = dict(lse=lse, slopes=torch.tensor([0.75], device=DEV), window=window)
    t = words(new, np.random.default_rng(1)) if tree else None
    out = c.attend_tree(q.to(DEV), ints([L]), t.to(DEV), **how) if tree else c.attend(q.to(DEV), ints([L]), **how)
    # (only differences of positions count)
    near_attend(out, lse, *attend64(q, key, val, 8 ** -0.5, slopes=torch.tensor([0.75]), window=window, tree=t), BF)


@pytest.mark.parametrize("group", [1, 8])
def test_bits_behind_a_drafts_tokens_count_nothing(group):
    """A word of ones: the token sees the whole draft, whose tokens are fewer."""
    new, ctx = [6, 2, 9], [200, 0, 90]
    c, lens, kvs, q = case(BF, group, 1, 64, new, ctx)
    tree = torch.full((sum(new),), -1, dtype=torch.int64)
    own = torch.cat([torch.full((m,), (1 << m) - 1, dtype=torch.int64) for m in new])
    opt = dict(slopes=torch.tensor([0.5] * group), window=30)
    how = dict(starts=torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=DEV), max_new=9, window=30,
               slopes=opt["slopes"].to(DEV))
    want, _ = check(c, lens, new, kvs, q, tree=own, **opt)
    assert torch.equal(c.attend_tree(q.to(DEV), ints(lens), tree.to(DEV), **how), want)


def test_one_token_has_no_stride():
    """Whatever lies between tokens does not matter where there is one."""
    from kv_plain import read_rows
    c, lens, kvs, q = case(BF, 4, 2, 64, [1], [20])
    want = c.attend(q.to(DEV), ints(lens))
    odd = lambda x, s: torch.as_strided(x, x.shape, (s, x.shape[2], 1))  # noqa: E731
    assert torch.equal(c.attend(odd(q.to(DEV), 259), ints(lens)), want)
    out = odd(torch.zeros(1, 4, 64, dtype=BF, device=DEV), 1)
    c.attend(q.to(DEV), ints(lens), out=out)
    assert torch.equal(out, want)
    k = torch.randn(1, 2, 64, device=DEV).to(BF)
    c.append(odd(k, 3), odd(k, 5), ints(lens), q=odd(q.to(DEV), 7), q_out=out)
    assert torch.equal(read_rows(c, 0, 0, lens[0])[:, -1], k.expand(2, 2, 64)) and torch.equal(out, q.to(DEV))


@pytest.mark.parametrize("n", [1, 5])
def test_queries_in_place_beside_their_keys_and_values(n):
    """In one fused projection's rows; keys and values that lie in the queries' own rows
    would be read while they are written, and are refused."""
    from kv_plain import read_rows
    from paper_2607_26566_gb300 import T2IError
    c, lens, _, _ = case(BF, 4, 2, 64, [n], [20])
    x = torch.randn(n + 1, (4 + 2 * 2) * 64, device=DEV).to(BF)
    q, k, v = (y.view(-1, h, 64) for y, h in zip(x.split([256, 128, 128], 1), (4, 2, 2)))
    L, w = ints(lens), torch.rand(64, device=DEV) + 0.5
    want = c.append(k[:n], v[:n], L, q=q[:n], q_norm=w)
    before = c.store.pool.clone(), x.clone()
    bad = [(q[:n, :2], v[:n]), (k[:n], q[:n, 2:]), (q[:n, 1:3], v[:n])]
    if n > 1:
        bad += [(q[1:n + 1, :2], v[:n]), (k[:n].contiguous(), x.view(-1)[64 * 8 * n - 256 - 64:][:n * 128].view(n, 2, 64))]
    for kk, vv in bad:
        with pytest.raises(T2IError, match="INVALID.*overlaps k or v"):
            c.append(kk, vv, L, q=q[:n], q_out=q[:n], q_norm=w)
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before[0]) and torch.equal(x, before[1])
    assert c.append(k[:n], v[:n], L, q=q[:n], q_out=q[:n], q_norm=w) is not None
    assert torch.equal(q[:n], want) and torch.equal(x[n], before[1][n]) and torch.equal(k, before[1][:, 256:384].view(-1, 2, 64))
    assert torch.equal(read_rows(c, 0, 0, lens[0])[:, -n:], torch.stack([k[:n], v[:n]]))


def test_a_gradient_is_not_lost_without_a_word():
    c, lens, kvs, q = case(BF, 4, 2, 64, [2], [20])
    q, L = q.to(DEV), ints(lens)
    kv = torch.zeros(2, 2, 64, dtype=BF, device=DEV)
    grad = lambda x: x.clone().requires_grad_()  # noqa: E731
    w = torch.ones(64, device=DEV)
    calls = (lambda: c.attend(grad(q), L), lambda: c.append(grad(kv), kv, L), lambda: c.append(kv, grad(kv), L),
             lambda: c.append(kv, kv, L, q=grad(q)), lambda: c.append(kv, kv, L, k_norm=grad(w)),
             lambda: c.attend(q, L, slopes=grad(w[:4])))
    before = c.store.pool.clone()
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before)
    for off in (torch.no_grad, torch.inference_mode):
        want = c.attend(q, L)  # (the appends below change the cache)
        with off():
            assert torch.equal(c.attend(grad(q), L), want)
            for call in calls:
                call()
    assert torch.equal(c.attend(grad(q).detach(), L), c.attend(q, L))


def test_a_table_row_ends_before_slots_cannot_be_counted():
    """Tiles end at multiples of 128 slots, and 2^31 is none that 32 bits count."""
    from paper_2607_26566_gb300 import T2IError
    c, lens, kvs, q = case(BF, 1, 1, 8, [1], [20], page=256)
    assert c.page_tokens == 8
    want = c.attend(q.to(DEV), ints(lens))
    most = (2 ** 31 - 256) // 8
    table = torch.empty(1, most + 31, dtype=torch.int32, device=DEV)
    table[:, :c.max_pages] = c.table
    assert torch.equal(c.attend(q.to(DEV), ints(lens), table=table[:, :most]), want)
    for pages in (most + 1, most + 31):
        with pytest.raises(T2IError, match="INVALID.*2\\^31 - 256"):
            c.attend(q.to(DEV), ints(lens), table=table[:, :pages])
