"""Arrays of weigh and select that share bytes (marked gpu): refused, with nothing launched, wherever a block would read or
write what another writes; arrays that lie side by side are not."""
import ctypes as C

import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_plain import DEV
from test_gpu_kv import BF, case, ints
from test_gpu_kv_weigh import WeighDesc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def refused(c, match, call):
    before = c.store.stats()["launches"]
    with pytest.raises(T2IError, match=match):
        call()
    assert c.store.stats()["launches"] == before


def test_weights_over_what_a_call_reads():
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1], [9, 9])
    q, lse = q.to(DEV), torch.zeros(2, 4, device=DEV)
    room = torch.zeros(1024, device=DEV)
    w, i = room[:80].view(2, 2, 20), room.view(torch.int32)
    for at in (0, 40, 78):
        refused(c, "lens.*overlaps weights", lambda: c.weigh(q, i[at:at + 2], lse, w))
        refused(c, "starts.*overlaps weights", lambda: c.weigh(q, ints(lens), lse, w, starts=i[at:at + 3], max_new=1))
        refused(c, "spans.*overlaps weights", lambda: c.weigh(q, ints(lens), lse, w, spans=i[at:at + 4].view(2, 2)))
        refused(c, "slopes.*overlaps weights", lambda: c.weigh(q, ints(lens), lse, w, slopes=room[at:at + 4]))
        refused(c, "table.*overlaps weights", lambda: c.weigh(q, ints(lens), lse, w, table=i[at:at + 4].view(2, 2)))
    refused(c, "lse.*overlaps weights", lambda: c.weigh(q, ints(lens), room[72:80].view(2, 4), w))
    refused(c, "q.*overlaps weights", lambda: c.weigh(room.view(BF)[128:640].view(2, 4, 64), ints(lens), lse, w))
    # behind them it is fine
    i[80:82] = ints(lens)
    assert c.weigh(q, i[80:82], lse, w) is w


def test_a_workspace_over_what_a_call_reads_or_writes(lib):
    """From C, where a caller brings the workspace."""
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1], [9, 9])
    need = C.c_uint64()
    assert lib.t2i_kv_weigh_workspace_bytes(c._h, 2, 2, C.byref(need)) == 0
    room = torch.zeros((need.value + 511) // 256 * 256, dtype=torch.uint8, device=DEV)
    base = (room.data_ptr() + 255) // 256 * 256
    q, L, starts = q.to(DEV), ints(lens), ints([0, 1, 2])
    lse, w = torch.zeros(2, 4, device=DEV), torch.zeros(2, 2, 20, device=DEV)
    spans, slopes = torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.zeros(4, device=DEV)
    good = dict(table=c.table.data_ptr(), lens=L.data_ptr(), starts=starts.data_ptr(), q=q.data_ptr(), lse=lse.data_ptr(),
                weights=w.data_ptr(), spans=spans.data_ptr(), slopes=slopes.data_ptr())
    how = dict(table_stride=c.max_pages, table_pages=c.max_pages, n_seqs=2, n_tokens=2, max_new=1, q_stride=256, seq_stride=40,
               head_stride=20, q_heads=4, n_slots=20, scale=0.125, decay=1.0, workspace=base, workspace_bytes=need.value)
    before = c.store.stats()["launches"]
    for name in good:
        d = WeighDesc(**{**good, **how, name: base + need.value // 512 * 256})
        assert lib.t2i_kv_weigh(c._h, C.byref(d), None) == 1, name
        assert name in c.store.last_error() and "overlap" in c.store.last_error(), c.store.last_error()
    assert c.store.stats()["launches"] == before
    assert lib.t2i_kv_weigh(c._h, C.byref(WeighDesc(**good, **how)), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()


def test_outputs_of_a_choice_over_one_another():
    c, lens, _, _ = case(BF, 4, 2, 64, [1, 1], [9, 9])
    w, kept = torch.rand(2, 2, 20, device=DEV), torch.zeros(2, 2, 5, dtype=torch.int32, device=DEV)
    room = torch.zeros(1024, device=DEV)
    out, i = room[:20].view(2, 2, 5), room.view(torch.int32)
    for at in (0, 7, 19):
        refused(c, "weights_out overlaps counts",
                lambda: c.select(w, ints(lens), 5, kept=kept, counts=i[at:at + 2], weights_out=out))
    refused(c, "weights_out overlaps kept", lambda: c.select(w, ints(lens), 5, kept=i[19:39].view(2, 2, 5), weights_out=out))
    c.select(w, ints(lens), 5, kept=kept, counts=i[20:22], weights_out=out)          # behind them
    assert i[20:22].tolist() == [5, 5] and torch.equal(out, torch.gather(w, 2, kept.long()))
