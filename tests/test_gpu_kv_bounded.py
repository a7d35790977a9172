"""A cache that stays bounded (marked gpu): attention, its weights, the choice and the eviction together, as a decoding
loop runs them, captured into a graph, and on streams of their own."""
import math

import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_bounded import attend64, near_weights, select_plain, weigh64
from kv_plain import DEV, make_cache, near_attend, read_rows, rows_of
from test_gpu_kv import BF, HF, case, gen, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


@pytest.mark.parametrize("dtype,window,sinks", [(BF, 0, 2), (HF, 0, 0), (BF, 30, 3)])
def test_a_loop_whose_cache_stays_bounded(dtype, window, sinks):
    """Prompts, then tokens; whenever a sequence is `slack` over its budget the slots of least attention go, in each
    layer and head others. Each call is compared with a plain form on what the cache then holds."""
    heads, kv, dim, layers, budget, slack, recent = 8, 2, 64, 2, 48, 6, 8
    lens = [37, 5, 90]
    c = make_cache(kv, dim, dtype, lens, layers=layers, more=60)
    g = gen(4)
    weights = [torch.zeros(3, kv, max(lens) + 60, device=DEV) for _ in range(layers)]
    new, evictions = list(lens), 0
    for step in range(24):
        n = sum(new)
        how = dict(starts=starts_of(new), max_new=max(new))
        for layer in range(layers):
            q = (2 * torch.randn(n, heads, dim, generator=g)).to(dtype)
            k, v = (torch.randn(n, kv, dim, generator=g).to(dtype).to(DEV) for _ in range(2))
            c.append(k, v, ints(lens), layer=layer, **how)
            lse = torch.full((n, heads), math.nan, device=DEV)
            opt = dict(window=window, sinks=sinks) if window else {}
            out = c.attend(q.to(DEV), ints(lens), lse=lse, layer=layer, **how, **opt)
            held = weights[layer].cpu()
            c.weigh(q.to(DEV), ints(lens), lse, weights[layer], layer=layer, decay=0.9, **how, **opt)
            got, at = weights[layer].cpu(), 0
            for s, (m, L) in enumerate(zip(new, lens)):
                w = slice(at, at + m)
                key, val = read_rows(c, s, layer, L).cpu()
                near_attend(out[w], lse[w], *attend64(q[w], key, val, dim ** -0.5, **opt), dtype, f"step {step}, sequence {s}")
                want, off = weigh64(q[w], key, lse[w].cpu(), dim ** -0.5, **opt)
                near_weights(got[s, :, :L], held[s, :, :L], want, off, L - m, 0.9, f"step {step}, sequence {s}")
                at += m
        if max(lens) > budget + slack:
            evictions += 1
            for layer in range(layers):
                before = [read_rows(c, s, layer, L).clone() for s, L in enumerate(lens)]
                w = weights[layer].cpu()
                kept, counts = c.select(weights[layer], ints(lens), budget, weights_out=weights[layer], recent=recent, sinks=sinks)
                c.evict(kept, counts, layer=layer)
                for s, L in enumerate(lens):
                    stay = min(L, budget)
                    assert int(counts[s]) == stay
                    after = read_rows(c, s, layer, stay)
                    for h in range(kv):
                        want = select_plain(w[s, h, :L].tolist(), stay, sinks, recent)
                        assert kept[s, h, :stay].tolist() == want
                        assert torch.equal(after[:, :, h], before[s][:, want, h])
                        assert torch.equal(weights[layer][s, h, :stay].cpu(), w[s, h][want])
            lens = [min(L, budget) for L in lens]
        new = [1, 1, 1]
        lens = [L + 1 for L in lens]
    assert evictions >= 3


@pytest.mark.parametrize("new", [[1, 1, 1], [24, 3, 32], [300, 40, 200]])
def test_a_graph_of_all_calls(new):
    """Captured once, replayed with other queries, lengths and weights: what eager calls give."""
    ctx = [700, 130, 300]
    c, lens, kvs, q = case(BF, 8, 2, 64, new, ctx)
    pool, n = c.store.pool.clone(), sum(new)
    q, L = q.to(DEV), ints(lens)
    how = dict(starts=starts_of(new), max_new=max(new), window=200, sinks=4)
    w = torch.rand(3, 2, max(lens), device=DEV)
    out, lse = torch.empty_like(q), torch.empty(n, 8, device=DEV)
    kept, counts = torch.zeros(3, 2, 64, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)

    def calls():
        c.attend(q, L, out=out, lse=lse, **how)
        c.weigh(q, L, lse, w, decay=0.5, **how)
        c.select(w, L, 64, kept=kept, counts=counts, weights_out=w, recent=8, sinks=4)
        c.evict(kept, counts)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.hold()
        calls()                                   # (loads the kernels)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
        for rep in range(3):
            other = (2 * torch.randn(q.shape, generator=gen(rep))).to(BF).to(DEV)
            lengths = ints([x - 7 * rep for x in lens])
            weights = torch.rand(w.shape, generator=gen(rep)).to(DEV)
            results = []
            for run in (calls, graph.replay):
                q.copy_(other), L.copy_(lengths), w.copy_(weights), c.store.pool.copy_(pool), kept.zero_()
                run()
                torch.cuda.synchronize()
                results.append([x.clone().view(torch.uint8) for x in (out, lse, w, kept, counts, c.store.pool)])
            assert all(torch.equal(a, b) for a, b in zip(*results)), rep


def test_calls_on_streams_side_by_side():
    """Two streams weigh and select at once, on caches of their own; and beside a busy stream each waits for its own only."""
    cases = [case(BF, 8, 2, 64, [300, 40], [500, 200], seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]

    def run(i, stream):
        c, lens, _, q = cases[i]
        with torch.cuda.stream(stream):
            c.hold()
            qd, L = q.to(DEV), ints(lens)
            lse = torch.zeros(340, 8, device=DEV)
            w = torch.zeros(2, 2, max(lens), device=DEV)
            got = []
            for _ in range(20):
                c.attend(qd, L, lse=lse, starts=starts_of([300, 40]), max_new=300)
                c.weigh(qd, L, lse, w, starts=starts_of([300, 40]), max_new=300, decay=0.0)
                got.append((w.clone(), *c.select(w, L, 50, recent=4)))
            return got

    alone = [run(i, torch.cuda.current_stream()) for i in range(2)]
    torch.cuda.synchronize()
    both = [run(i, streams[i]) for i in range(2)]
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for x, y in zip(a, b):
            assert all(torch.equal(u, v) for u, v in zip(x, y))


def test_an_output_belongs_to_the_stream_that_writes_it():
    c, lens, _, _ = case(BF, 4, 2, 64, [1, 1], [300, 20])
    w = torch.rand(2, 2, max(lens), device=DEV)
    want = c.select(w, ints(lens), 30)
    side = torch.cuda.Stream()
    L = ints(lens)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    kept, counts = c.select(w, L, 30, stream=side)
    again = torch.zeros_like(kept)       # of the current stream: other memory, whatever `side` still does
    assert again.data_ptr() != kept.data_ptr()
    side.synchronize()
    assert torch.equal(counts, want[1]) and counts.tolist() == [30, 21]
    assert torch.equal(kept[0], want[0][0]) and torch.equal(kept[1, :, :21], want[0][1, :, :21])  # (behind them: anything)


def test_pages_beyond_4_gib():
    """Keys and rows at offsets that pass 32 bits."""
    c = make_cache(1, 128, BF, [40, 70], page=1 << 30, spare=4)
    T = c.page_tokens
    table = torch.tensor([[5], [4]], dtype=torch.int32, device=DEV)
    rows = rows_of(c)
    g = gen(0)
    lens, new = [40, 70], [1, 1]
    kvs = [tuple(torch.randn(L, 1, 128, generator=g).to(BF) for _ in range(2)) for L in lens]
    for s, page in enumerate((5, 4)):
        for i in range(2):
            rows[page, 0, i, :, :lens[s]] = kvs[s][i].transpose(0, 1).to(DEV)
    assert T > 70
    q = torch.randn(2, 4, 128, generator=g).to(BF)
    lse = torch.zeros(2, 4)
    for s in range(2):
        lse[s] = attend64(q[s:s + 1], *kvs[s], 128 ** -0.5)[1][0].float()
    w = torch.zeros(2, 1, 70, device=DEV)
    c.weigh(q.to(DEV), ints(lens), lse.to(DEV), w, table=table, max_len=70)
    for s in range(2):
        want, off = weigh64(q[s:s + 1], kvs[s][0], lse[s:s + 1], 128 ** -0.5)
        near_weights(w[s, :, :lens[s]].cpu(), torch.zeros(1, lens[s]), want, off, lens[s] - 1, 1.0)
    kept, counts = c.select(w, ints(lens), 20)
    c.evict(kept, counts, table=table)
    for s, page in enumerate((5, 4)):
        for i in range(2):
            assert torch.equal(rows[page, 0, i, 0, :20].cpu(), kvs[s][i][kept[s, 0].cpu().long(), 0])


def test_far_slots_of_a_long_cache():
    """Slots beyond 2^24, which fp32 does not count, and offsets of weights beyond 2^31 bytes."""
    dim, far = 8, (1 << 25) + 777
    c = make_cache(1, dim, BF, [far + 40], page=1 << 30, fill=0)
    T = c.page_tokens
    g = gen(3)
    key = torch.randn(60, 1, dim, generator=g).to(BF)
    rows, pages = rows_of(c), c.pages(0)
    slots = torch.arange(far - 20, far + 40)
    for j, k in zip(slots.tolist(), key):
        rows[pages[j // T], 0, 0, :, j % T] = k.to(DEV)
    q = torch.randn(3, 2, dim, generator=g).to(BF)
    L, window = far + 40, 30
    slopes = torch.tensor([0.5, 0.125])
    plain = dict(slopes=slopes, window=window)
    lse = attend64(q, key, key, 1.0, **plain)[1].float()
    w = torch.zeros(1, 1, L, device=DEV)
    c.weigh(q.to(DEV), ints([L]), lse.to(DEV), w, scale=1.0, slopes=slopes.to(DEV), window=window)
    want, off = weigh64(q, key, lse, 1.0, **plain)
    near_weights(w[0, :, far - 20:].cpu(), torch.zeros(1, 60), want, off, 57, 1.0)
    assert (w[0, :, :far - 20] == 0).all()
    w[0, 0, :far - 20] = 1e-3 * torch.rand(far - 20, device=DEV)
    kept, counts = c.select(w, ints([L]), 32, recent=5)
    order = torch.sort(w[0, 0, :L - 5], descending=True, stable=True).indices[:27]
    assert kept[0, 0].tolist() == sorted(order.tolist()) + list(range(L - 5, L)) and counts.tolist() == [32]
    before = [[rows[pages[j // T], 0, i, 0, j % T].clone() for j in kept[0, 0].tolist()] for i in range(2)]
    c.evict(kept, counts)
    for i in range(2):
        assert torch.equal(rows[pages[0], 0, i, 0, :32], torch.stack(before[i]))


@pytest.mark.parametrize("call", ["select", "evict"])
def test_a_wait_that_ran_out_is_reported_by_the_next_call(call):
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1], [30, 20])
    w = torch.zeros(2, 2, 31, device=DEV)
    kept, counts = c.select(w, ints(lens), 10)
    c.inject_timeout(1)
    c.weigh(q.to(DEV), ints(lens), torch.zeros(2, 4, device=DEV), w)
    torch.cuda.synchronize()
    with pytest.raises(T2IError, match="CUDA.*" + call + ".*gave up"):
        c.select(w, ints(lens), 10) if call == "select" else c.evict(kept, counts)
    c.evict(kept, counts)
    c.close()
    for again in (lambda: c.select(w, ints(lens), 10, kept=kept, counts=counts), lambda: c.evict(kept, counts)):
        with pytest.raises(ValueError, match="closed"):
            again()
