"""The choice of what stays in rows around what a cluster's registers hold (marked gpu): 131,072 slots, 16 a thread of eight
blocks of 1,024. A longer row, or one that is longer than its caller said, is read from memory in each pass."""
import pytest
import torch

from test_gpu_kv_evict import any_cache, check, some  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
HELD = 131_072


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("length", [HELD - 1, HELD, HELD + 1, HELD + 4097])
@pytest.mark.parametrize("keep", [1, 30_000])
def test_the_longest_row_that_is_held_and_the_next(any_cache, length, keep, in_place):  # noqa: F811
    check(any_cache, some(1, 2, HELD + 4097, length, 64), [length], keep, recent=50, sinks=4, in_place=in_place)


@pytest.mark.parametrize("max_len", [2048, 2049, 8192, 8193, 16_384, 16_385])
@pytest.mark.parametrize("length", [2047, 2048, 2049, 8192, 8193, 16_384, 16_385])
def test_rows_around_what_a_block_holds(any_cache, max_len, length):  # noqa: F811
    """2, 8 and 16 slots a thread, going by max_len, of many rows (a block each) and of few (several)."""
    for n in (1, 160):
        check(any_cache, some(n, 1, 16_385, length, 32), [length] * n, 1000, recent=3, sinks=3, max_len=max_len)
