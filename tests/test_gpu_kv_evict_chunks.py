"""Rows moved together in lists of several chunks (marked gpu): a chunk's length depends on the width of a head and on how
its columns are shared out, so lists end just before, at and behind one chunk and two in each form. The whole pool is
compared, what no row uses included."""
import pytest
import torch

from kv_plain import DEV, rows_of
from test_gpu_kv import BF, ints
from test_gpu_kv_evict import lists, random_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def check(c, lens, counts, seed):
    kept = lists(lens, counts, c.kv_heads, seed)
    want = c.store.pool.clone()
    T, rows, size = c.page_tokens, rows_of(c), c.store.page_bytes // 2
    shape = rows.shape[1:]
    new = want.view(c.dtype).view(-1, size)[:, :shape.numel()].view(-1, *shape).view(torch.int16)
    old = rows.view(torch.int16)
    for s, n in enumerate(counts):
        pages, dst = torch.tensor(c.pages(s), dtype=torch.long, device=DEV), torch.arange(n, device=DEV)
        for h in range(c.kv_heads):
            src = kept[s, h, :n].long().to(DEV)
            for layer in range(c.layers):
                new[pages[dst // T], layer, :, h, dst % T] = old[pages[src // T], layer, :, h, src % T]
    c.evict(kept.to(DEV), ints(counts))
    assert torch.equal(c.store.pool, want)


# chunks are of 64 to 512 rows: 4 x (256 threads / columns of a block)
COUNTS = [1, 63, 64, 65, 127, 129, 255, 256, 257, 339, 340, 341, 511, 512, 513, 680, 681, 1023, 1024, 1025]


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 64, 80, 120, 128])
def test_few_lists(dim):
    """Their columns are shared out where a row has four vectors or more."""
    counts = COUNTS + [2000, 2047, 2049, 5000]
    lens = [n + n // 2 + 1 for n in counts]
    check(random_cache(1, dim, BF, lens, 65536), lens, counts, dim)


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 80, 120, 128])
def test_many_lists(dim):
    """More than the GPU has places for blocks: each moves whole rows."""
    counts = [n for n in COUNTS if n <= 1100] if dim <= 16 else [min(n, 3 * 1024 // (dim // 8) // 4) for n in COUNTS]
    lens = [n + n // 3 + 2 for n in counts]
    check(random_cache(8, dim, BF, lens, 262144, layers=4), lens, counts, dim)
