"""The key/value cache's beginning and end (marked gpu): handles, pages and stores that
are closed in any order."""
import pytest
import torch

from paper_2607_26566_gb300 import KVCache, Store
from kv_plain import DEV, make_cache
from test_gpu_kv import BF, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def every_call(c):
    x = torch.zeros(1, 1, 64, dtype=BF, device=DEV)
    one = ints([1])
    return (lambda: c.append(x, x, one), lambda: c.attend(x, one), lambda: c.commit(one, one.view(1, 1), one),
            lambda: c.attend_tree(x, one, torch.ones(1, dtype=torch.int64, device=DEV)), lambda: c.reserve([50]),
            lambda: c.release([0]), c.refresh, c.hold, lambda: c.inject_timeout(1))


def test_a_store_closed_before_its_caches_closes_them():
    a = make_cache(1, 64, BF, [10])
    b = KVCache(a.store, 1, 64, max_tokens=100)
    gone = KVCache(a.store, 1, 64, max_tokens=100)
    del gone
    a.store.close()
    for c in (a, b):
        for call in every_call(c):
            with pytest.raises(ValueError, match="closed"):
                call()
        c.close()
    a.store.close()


def test_a_closed_cache_takes_no_pages():
    c = make_cache(1, 64, BF, [10])
    c.close()
    assert c.store.stats()["used_pages"] == 0
    for call in every_call(c):
        with pytest.raises(ValueError, match="closed"):
            call()
    assert c.store.stats()["used_pages"] == 0
    c.close()


def test_a_sequence_that_is_none_is_not_released():
    """(Python would count -1 from the end, and the page table keep what was freed.)"""
    c = make_cache(1, 64, BF, [10, 20])
    pages, table = [c.pages(0), c.pages(1)], c.table.clone()
    for seqs in ([-1], [2], [0, -2], [0, 5]):
        with pytest.raises(ValueError, match="outside the cache"):
            c.release(seqs)
    assert [c.pages(0), c.pages(1)] == pages and torch.equal(c.table, table)
    c.release([1, 1])
    assert c.pages(1) == [] and (c.table[1] == -1).all() and torch.equal(c.table[0], table[0])


@pytest.mark.parametrize("where", ["full", "cache"])
def test_a_cache_that_cannot_be_made_leaves_nothing(monkeypatch, where):
    from paper_2607_26566_gb300 import kv

    class Counting:
        def __init__(self, lib):
            self.lib, self.handles = lib, 0

        def __getattr__(self, name):
            f = getattr(self.lib, name)
            return {"t2i_kv_create": lambda *a: self.made(f(*a)), "t2i_kv_destroy": lambda h: self.gone(f(h))}.get(name, f)

        def made(self, st):
            self.handles += st == 0
            return st

        def gone(self, st):
            self.handles -= 1
            return st

    def fails(*a, **k):
        raise MemoryError("none left")

    store = Store(torch.empty(64 << 16, dtype=torch.uint8, device=DEV), 1 << 16)
    lib = Counting(kv.L.load())
    with monkeypatch.context() as m:
        m.setattr(kv.L, "load", lambda: lib)
        KVCache(store, 2, 64).close()
        assert lib.handles == 0
        m.setattr(kv.torch if where == "full" else kv._kv, where, fails)
        with pytest.raises(MemoryError):
            KVCache(store, 2, 64)
    assert lib.handles == 0 and not list(store._users)
