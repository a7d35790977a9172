"""An attention whose waits run out (marked gpu): its kernels end, touch nothing that
is not theirs, and the next call reports it. The loads are left out on request, so
that the bounded waits for them run their second."""
import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_plain import DEV
from test_gpu_kv import BF, HF, case, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


@pytest.mark.parametrize("dtype,new", [(BF, [1, 1, 1]), (HF, [40, 1, 300])])
@pytest.mark.parametrize("next_call", ["attend", "append", "commit"])
def test_a_wait_that_runs_out_is_reported_and_harms_nothing(dtype, new, next_call):
    c, lens, _, q = case(dtype, 8, 2, 128, new, [3000, 50, 1500])
    n = sum(new)
    q, L = q.to(DEV), ints(lens)
    how = dict(starts=starts_of(new), max_new=max(new))
    want = c.attend(q, L, **how)
    before = c.store.pool.clone()
    around = torch.full((n + 64, 8, 128), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((n + 64, 8), 7.0, device=DEV)
    used = torch.full((64 << 20,), 1, dtype=torch.uint8, device=DEV)  # what the workspace finds: notes that look valid
    torch.cuda.synchronize()
    del used
    c.inject_timeout(2)
    assert torch.equal(c.attend(q, L, **how), want)                   # the first one has its loads
    c.attend(q, L, out=around[32:32 + n], lse=lse[32:32 + n], **how)
    torch.cuda.synchronize()
    for x in (around, lse):
        assert (x[:32] == 7).all() and (x[32 + n:] == 7).all()
    assert torch.equal(c.store.pool, before)

    kv = torch.zeros(n, 2, 128, dtype=dtype, device=DEV)
    calls = dict(attend=lambda: c.attend(q, L, **how), append=lambda: c.append(kv, kv, L, **how),
                 commit=lambda: c.commit(L, torch.ones(3, 1, dtype=torch.int32, device=DEV), ints([1, 1, 1])))
    with pytest.raises(T2IError, match="CUDA.*" + next_call + ".*gave up"):
        calls[next_call]()
    torch.cuda.synchronize()
    assert torch.equal(c.store.pool, before)                           # it did nothing
    assert torch.equal(c.attend(q, L, **how), want)                    # reported once


def test_a_null_handle_is_refused(lib):
    from paper_2607_26566_gb300 import _lib as L
    assert lib.t2i_kv_inject_timeout(None, 1) == L.ERR_INVALID
