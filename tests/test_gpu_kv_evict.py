"""What stays of a cache, and its rows moved together (marked gpu): whole numbers and bits, equal to a plain form's."""
import math

import numpy as np
import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_bounded import select_plain
from kv_plain import DEV, make_cache, rows_of
from test_gpu_kv import BF, HF, gen, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


@pytest.fixture(scope="module")
def any_cache():
    return make_cache(2, 64, BF, [8])


def check(c, w, lens, keep, recent=0, sinks=0, keeps=None, in_place=False, max_len=0, slots=None):
    """select on weights [sequences, heads, slots] (on the host)."""
    n, heads, W = w.shape
    width = min(keep, W)
    kept = torch.full((n, heads, width + 2), -7, dtype=torch.int32, device=DEV)
    counts = torch.full((n,), -7, dtype=torch.int32, device=DEV)
    d = w.clone().to(DEV)
    out = d if in_place else torch.full((n, heads, width + 3), -7.0, device=DEV)
    before = out.clone()
    c.select(d, ints(lens), keep, kept=kept, counts=counts, weights_out=out, recent=recent, sinks=sinks,
             keeps=None if keeps is None else ints(keeps), max_len=max_len)
    kept, counts, out, before = kept.cpu(), counts.cpu(), out.cpu(), before.cpu()
    for s in range(n):
        L = lens[s] if 0 <= lens[s] <= W else 0
        stay = min(L, keep, max(keeps[s], 0) if keeps else keep)
        assert int(counts[s]) == stay
        for h in range(heads):
            want = select_plain(w[s, h, :L].tolist(), stay, sinks, recent)
            assert kept[s, h, :stay].tolist() == want, (s, h)
            assert (kept[s, h, stay:] == -7).all()
            assert torch.equal(out[s, h, :stay].view(torch.int32), w[s, h][want].view(torch.int32))
            assert torch.equal(out[s, h, stay:].view(torch.int32), before[s, h, stay:].view(torch.int32))
    if not in_place:
        assert torch.equal(d.cpu().view(torch.int32), w.view(torch.int32))


def some(n, heads, W, seed=0, values=0):
    g = gen(seed)
    w = torch.exp(2 * torch.randn(n, heads, W, generator=g))
    w[torch.rand(w.shape, generator=g) < 0.1] = 0
    return (w * values).floor() / values if values else w


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("recent,sinks", [(0, 0), (5, 3), (1000, 0), (0, 1000), (30, 30)])
@pytest.mark.parametrize("keep", [1, 17, 40, 300])
def test_select(any_cache, keep, recent, sinks, in_place):
    lens = [0, 1, 16, 17, 18, 39, 41, 299, 300, 301, 513, 600]
    check(any_cache, some(len(lens), 2, 600), lens, keep, recent, sinks, in_place=in_place)


@pytest.mark.parametrize("values", [1, 2, 8])
@pytest.mark.parametrize("keep", [3, 100, 1500, 2047])
def test_equal_weights_go_by_slot(any_cache, keep, values):
    check(any_cache, some(3, 2, 2049, values, values), [2049, 2048, 1700], keep, recent=1, sinks=2)
    check(any_cache, torch.zeros(1, 1, 2049), [2049], keep, in_place=True)


def test_any_bits(any_cache):
    """Every kind of number: infinities, NaN of either sign, subnormal ones, zeros of either sign, negative ones."""
    g = np.random.default_rng(0)
    w = g.integers(0, 1 << 32, (4, 3, 5000), dtype=np.uint64).astype(np.uint32)
    special = np.array([0, 1 << 31, 0x7F800000, 0xFF800000, 0x7FC00000, 0xFFC00001, 1, 0x80000001, 0x7F7FFFFF, 0xFF7FFFFF], np.uint32)
    w[:, 1] = special[g.integers(0, len(special), (4, 5000))]
    w[:, 2] = (w[:, 2] & 0x1FF) | 0x3F800000      # alike in their leading bits
    w = torch.from_numpy(w.view(np.float32).copy())
    for keep in (1, 700, 2500, 4990):
        check(any_cache, w, [5000, 4999, 4500, 10], keep, sinks=1, recent=1)


@pytest.mark.parametrize("n,heads,W,lens,keep", [
    (1, 1, 100_000, [99_999], 5000), (1, 8, 33_000, [33_000], 8192), (2, 2, 200_001, [200_001, 70_000], 60_000),
    (300, 1, 900, None, 700)])
@pytest.mark.parametrize("in_place", [False, True])
def test_long_rows_and_many(any_cache, n, heads, W, lens, keep, in_place):
    lens = lens or [(i * 37) % (W + 1) for i in range(n)]
    check(any_cache, some(n, heads, W, W, 64), lens, keep, recent=100, sinks=4, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_a_row_that_no_cluster_holds(any_cache, in_place):
    """More slots than eight blocks' shared memory has room for."""
    check(any_cache, some(1, 2, 400_000, 3), [400_000], 100_000, recent=1000, sinks=16, in_place=in_place)


@pytest.mark.parametrize("max_len", [1, 100, 1 << 30])
def test_a_wrong_max_len_changes_no_result(any_cache, max_len):
    check(any_cache, some(2, 2, 90_000, 5, 16), [90_000, 3000], 2000, sinks=4, recent=9, max_len=max_len)
    check(any_cache, some(2, 2, 90_000, 5, 16), [90_000, 3000], 2000, in_place=True, max_len=max_len)


def test_fewer_of_some_and_lengths_that_make_no_sense(any_cache):
    w = some(6, 2, 500)
    check(any_cache, w, [500, 400, 300, -1, 501, 1 << 30], 200, recent=7, sinks=7, keeps=[200, 0, 11, 5, 5, 5])
    check(any_cache, w, [500, 400, 300, 200, 100, 0], 200, keeps=[-5, 1, 1 << 30, 200, 200, 9])
    check(any_cache, w, [500] * 6, 0)


def test_strides_shared_rows_and_made_outputs(any_cache):
    c = any_cache
    w = some(3, 4, 100, 7)
    wide = torch.full((3, 9, 130), math.nan, device=DEV)
    wide[:, 2:6, 20:120] = w.to(DEV)
    kept, counts = c.select(wide[:, 2:6, 20:120], ints([100, 50, 20]), 30, sinks=2)
    assert kept.shape == (3, 4, 30) and counts.tolist() == [30, 30, 20]
    assert kept[0, 3].tolist() == select_plain(w[0, 3].tolist(), 30, 2, 0)
    # one row read for two heads (permuted, too: any order of reading)
    kept, _ = c.select(w[:, :1].to(DEV).expand(3, 2, 100), ints([100] * 3), 10)
    assert torch.equal(kept[:, 0], kept[:, 1]) and kept[2, 1].tolist() == select_plain(w[2, 0].tolist(), 10, 0, 0)
    by_head = w.permute(1, 0, 2).contiguous().to(DEV).permute(1, 0, 2)
    kept, _ = c.select(by_head, ints([100] * 3), 10)
    assert kept[1, 2].tolist() == select_plain(w[1, 2].tolist(), 10, 0, 0)
    kept, counts = c.select(w.to(DEV), ints([100, 100, 3]), 1000)
    assert kept.shape == (3, 4, 100) and counts.tolist() == [100, 100, 3] and kept[1, 1].tolist() == list(range(100))


# ------------------------------------------------------------------ evict
def lists(lens, counts, heads, seed=0):
    g = np.random.default_rng(seed)
    out = np.full((len(lens), heads, max(max(counts), 1) + 2), -1, np.int32)
    for s, (L, n) in enumerate(zip(lens, counts)):
        for h in range(heads):
            out[s, h, :n] = np.sort(g.permutation(L)[:n])
    return torch.from_numpy(out)


def moved(c, before, kept, counts, layers):
    """The pool's rows after the call, from those before it."""
    want, T = before.clone(), c.page_tokens
    for s, n in enumerate(counts):
        pages = torch.tensor(c.pages(s), dtype=torch.long)
        dst = torch.arange(n)
        for h in range(c.kv_heads):
            src = kept[s, h, :n].long()
            for layer in layers:
                want[pages[dst // T], layer, :, h, dst % T] = before[pages[src // T], layer, :, h, src % T]
    return want


def random_cache(heads, dim, dtype, lens, page, layers=1):
    c = make_cache(heads, dim, dtype, lens, page=page, layers=layers)
    c.store.pool.copy_(torch.randint(0, 256, c.store.pool.shape, dtype=torch.uint8, generator=gen(dim)).to(DEV))
    return c


@pytest.mark.parametrize("heads,dim,layers,page", [(2, 128, 1, 65536), (1, 8, 3, 1024), (3, 80, 2, 65536), (8, 64, 1, 16384),
                                                   (1, 128, 1, 1 << 20), (2, 120, 1, 8192)])
def test_evict(heads, dim, layers, page):
    lens = [0, 1, 9, 100, 700, 1000, 513]
    counts = [0, 1, 4, 100, 300, 999, 1]
    c = random_cache(heads, dim, HF, lens, page, layers)
    kept = lists(lens, counts, heads, dim)
    before = rows_of(c).view(torch.int16).cpu().clone()
    pool = c.store.pool.clone()
    c.evict(kept.to(DEV), ints(counts), layer=layers - 1)
    assert torch.equal(rows_of(c).view(torch.int16).cpu(), moved(c, before, kept, counts, [layers - 1]))
    c.store.pool.copy_(pool)
    c.evict(kept.to(DEV), ints(counts))
    assert torch.equal(rows_of(c).view(torch.int16).cpu(), moved(c, before, kept, counts, range(layers)))


def test_one_list_for_all_heads_chosen_sequences_and_long_ones():
    lens, counts = [5000, 40, 20_000], [4000, 40, 9000]
    c = random_cache(2, 64, BF, lens, 65536)
    kept = lists(lens, counts, 1, 3)
    before = rows_of(c).view(torch.int16).cpu().clone()
    pick = [2, 0]
    c.evict(kept[pick].to(DEV).expand(-1, 2, -1), ints([counts[i] for i in pick]), table=c.table[pick])
    want = moved(c, before, kept.expand(-1, 2, -1), [counts[0], 0, counts[2]], [0])
    assert torch.equal(rows_of(c).view(torch.int16).cpu(), want)


def test_entries_that_make_no_sense_stay_in_bounds():
    c = random_cache(2, 64, BF, [100, 100], 65536)
    before = c.store.pool.clone()
    same = torch.arange(100, dtype=torch.int32).expand(2, 2, 100)
    c.evict(same.to(DEV), ints([100, 100]))                                    # every row in its place
    c.evict(same.to(DEV), ints([-3, 0]))
    c.evict(torch.full((2, 2, 50), -4, dtype=torch.int32, device=DEV), ints([50, 1 << 30]))
    c.evict(torch.full((2, 2, 50), 0x7FFFFFFF, dtype=torch.int32, device=DEV), ints([50, 50]))   # no such slots
    c.evict((same + 1).to(DEV), ints([100, 100]), table=torch.full((2, 7), -1, dtype=torch.int32, device=DEV))
    c.evict((same + 1).to(DEV), ints([100, 100]), table=torch.full((2, 7), 1 << 30, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before)


def test_refusals(any_cache):
    c = any_cache
    w, L = torch.zeros(2, 2, 20, device=DEV), ints([20, 9])
    kept, counts = torch.zeros(2, 2, 5, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)

    def no(error, match, call, *a, **k):
        before = c.store.stats()["launches"]
        with pytest.raises(error, match=match):
            call(*a, **k)
        assert c.store.stats()["launches"] == before

    no(ValueError, "gradient", c.select, w.clone().requires_grad_(), L, 5)
    no(TypeError, "dtype", c.select, w.half(), L, 5)
    no(TypeError, "dtype", c.select, w, L, 5, kept=kept.long())
    no(ValueError, "weights", c.select, w[0], L, 5, kept=kept, counts=counts)
    no(ValueError, "weights", c.select, w[0], L, 5)
    no(TypeError, "weights", c.select, None, L, 5)
    no(ValueError, "keep", c.select, w, L, -1)
    no(ValueError, "lens", c.select, w, L[:1], 5)
    no(ValueError, "kept", c.select, w, L, 6, kept=kept)
    no(ValueError, "kept", c.select, w, L, 5, kept=kept[:, :1])
    no(ValueError, "weights_out", c.select, w, L, 5, weights_out=w[..., :4])
    no(ValueError, "keeps", c.select, w, L, 5, keeps=counts[:1])
    no(ValueError, "keep", c.select, w, L, -1, kept=kept, counts=counts)
    no(ValueError, "recent", c.select, w, L, 5, recent=-1)
    no(T2IError, "overlap", c.select, w, L, 5, weights_out=w[..., 1:])         # weights, but not in their place
    no(T2IError, "overlap", c.select, w, L, 5, kept=kept[:1].expand(2, -1, -1))
    no(T2IError, "overlap", c.select, w[:1].expand(2, -1, -1), L, 5, weights_out=w[:1].expand(2, -1, -1))
    no(T2IError, "overlap", c.select, w, L, 5, kept=w.view(torch.int32)[..., :5])
    no(T2IError, "counts.*overlaps lens", c.select, w, L, 5, counts=L)          # (lens would change while it is read)
    no(T2IError, "counts.*overlaps lens", c.select, w, L, 5, keeps=counts, counts=counts)
    no(T2IError, "overlap", c.select, w, L, 5, counts=kept[0, 0, :2], kept=kept)
    no(T2IError, "overlap", c.select, w, L, 5, counts=w.view(torch.int32)[0, 0, :2])
    both = torch.zeros(22, dtype=torch.int32, device=DEV)
    no(T2IError, "kept.*overlaps lens", c.select, w, both[:2], 5, kept=both[:20].view(2, 2, 5))
    assert c.select(w[:0], L[:0], 5)[0].shape == (0, 2, 5)
    no(TypeError, "counts", c.evict, kept[:1], None)
    no(TypeError, "dtype", c.evict, kept[:1].long(), counts[:1])
    no(ValueError, "kept", c.evict, kept[:1, :1], counts[:1])
    no(ValueError, "kept", c.evict, kept[0], counts[:1])
    no(ValueError, "counts", c.evict, kept[:1], counts)
    no(ValueError, "more sequences", c.evict, kept, counts)
    no(T2IError, "layers", c.evict, kept[:1], counts[:1], layer=1)
    c.evict(kept[:0], counts[:0])
    c.evict(kept[:1, :, :0], counts[:1])


def test_thresholds_at_zero(any_cache):
    """Exactly the numbers from 0 (and -0) on stay, or from infinity on, or all but NaN, or some of the zeros."""
    g = np.random.default_rng(1)
    neg = -np.exp(g.standard_normal(300)).astype(np.float32)
    tiny = np.array([-1.4e-45, 1.4e-45, -1e-38, 1e-38], np.float32)
    rows = [np.concatenate([neg, np.zeros(40), -np.zeros(40), np.exp(g.standard_normal(100)), tiny, [math.inf] * 5,
                            [-math.inf] * 5, [math.nan] * 6]).astype(np.float32) for _ in range(4)]
    for r in rows:
        g.shuffle(r)
    w = torch.from_numpy(np.stack(rows))[None]
    L = w.shape[2]
    positive, zeros = 100 + 2 + 5, 80
    for keep in (5, positive, positive + 1, positive + 37, positive + zeros, positive + zeros + 1, L - 11, L - 6, L - 5, L - 1):
        check(any_cache, w, [L], keep)
        check(any_cache, w, [L], keep, in_place=True)
