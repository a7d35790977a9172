"""The key/value cache beside graphs, streams and threads (marked gpu)."""
import sys
import threading

import pytest
import torch

from paper_2607_26566_gb300 import KVCache, Store
from kv_plain import DEV
from test_gpu_kv import BF, case, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def split_case():
    """One token a sequence, and units in several runs: parts and notes in the workspace."""
    c, lens, _, q = case(BF, 8, 2, 128, [1, 1, 1], [3000, 50, 1500])
    return c, q.to(DEV), ints(lens)


def test_a_graph_writes_nothing_that_is_not_its_own():
    """Captured, then a far larger call on the same stream, then other tensors of all
    sizes: a replay gives the same output and leaves them alone."""
    c, q, lens = split_case()
    many = torch.randn(3 * 2000, 8, 128, device=DEV).to(BF)
    want = c.attend(q, lens)
    out = torch.zeros_like(want)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c.attend(q, lens)
    with torch.cuda.graph(graph, stream=s):
        c.attend(q, lens, out=out)
    with torch.cuda.stream(s):
        c.attend(many, lens, starts=starts_of([2000, 1, 1200]), max_new=2000)
    fill = []
    for stream in (torch.cuda.current_stream(), s):
        with torch.cuda.stream(stream):
            fill += [torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV) for n in (1 << 12, 1 << 20, 9 << 20, 40 << 20, 80 << 20)]
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert all((f == 0x5A).all() for f in fill)


def test_graphs_replayed_side_by_side():
    """Two graphs of one cache, captured one after the other where torch captures by
    default, share nothing."""
    c, q, lens = split_case()
    q2 = torch.randn_like(q)
    want = [c.attend(q, lens), c.attend(q2, lens)]
    graphs, outs = [], []
    for x in (q, q2):
        outs.append(torch.zeros_like(want[0]))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.attend(x, lens, out=outs[-1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(50):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_a_call_keeps_no_memory():
    c, q, lens = split_case()
    out = torch.empty_like(q)
    before = torch.cuda.memory_allocated()
    for s in (torch.cuda.current_stream(), torch.cuda.Stream()):
        c.attend(q, lens, out=out, stream=s)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


def test_threads_with_streams_of_their_own():
    """Four threads call one cache, each on streams that it has not seen before."""
    c, q, lens = split_case()
    want = c.attend(q, lens)
    torch.cuda.synchronize()
    bad, go = [], threading.Barrier(4)

    def work():
        try:
            go.wait()
            for _ in range(8):
                s = torch.cuda.Stream()
                with torch.cuda.stream(s):
                    got = [c.attend(q, lens) for _ in range(10)]
                s.synchronize()
                assert all(torch.equal(x, want) for x in got)
        except Exception as e:  # (an assert in a thread is not pytest's)
            bad.append(e)

    every = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=work) for _ in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(every)
    assert not bad, bad


def test_a_cache_made_on_a_busy_stream_is_ready_for_any():
    """The page table's first fill does not come after what another stream wrote to it."""
    store = Store(torch.empty(64 << 16, dtype=torch.uint8, device=DEV), 1 << 16)
    slow = torch.randn(4096, 4096, device=DEV)
    s = torch.cuda.Stream()
    for made in (None, s, s.cuda_stream, 0):
        torch.cuda.synchronize()
        for stream in (torch.cuda.current_stream(), s):
            with torch.cuda.stream(stream):
                for _ in range(10):
                    slow = slow @ slow.clamp(-1e-3, 1e-3)
        c = KVCache(store, 2, 64, max_seqs=2, max_tokens=400, stream=made)
        other = torch.cuda.Stream()
        c.reserve([300, 200], stream=other)
        with torch.cuda.stream(other):
            got = c.table.clone()
        torch.cuda.synchronize()
        for table in (got, c.table):  # as the reserving stream left it, and in the end
            assert [[p for p in row if p >= 0] for row in table.tolist()] == [c.pages(0), c.pages(1)]
        c.close()


def test_a_stream_argument_names_the_same_stream_everywhere():
    c, q, lens = split_case()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert c._stream(None) == s
        assert c._stream(0) == torch.cuda.default_stream(DEV)
        assert c._stream(s.cuda_stream).cuda_stream == s.cuda_stream
    assert c._stream(s) is s


def test_an_output_belongs_to_the_stream_that_writes_it():
    """What a call with a stream makes comes from that stream's memory and goes back to it."""
    c, q, lens = split_case()
    kv = torch.zeros(3, 2, 128, dtype=BF, device=DEV)
    one = torch.ones(3, dtype=torch.int64, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call in (lambda: c.attend(q, lens, stream=s), lambda: c.attend(q, lens, stream=s.cuda_stream),
                 lambda: c.attend_tree(q, lens, one, stream=s), lambda: c.append(kv, kv, lens, q=q, stream=s)):
        with torch.cuda.stream(s):
            mine = torch.empty_like(q)
        at = mine.data_ptr()
        del mine
        out = call()
        assert out.data_ptr() == at       # the block that the stream had free
        torch.cuda.synchronize()
        del out
        keep = [torch.empty_like(q) for _ in range(8)]
        assert all(x.data_ptr() != at for x in keep)
        with torch.cuda.stream(s):
            assert torch.empty_like(q).data_ptr() == at
