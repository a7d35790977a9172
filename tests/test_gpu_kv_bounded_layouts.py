"""Weights and lists that lie by head (marked gpu): [kv_heads, sequences, slots] in memory, as a caller that splits heads keeps
them, whose rows overlap no more than those that lie by sequence."""
import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_plain import DEV
from test_gpu_kv import BF, case, gen, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def by_head(x, room=0):
    """x [sequences, heads, slots] in memory [heads, sequences, slots + room]."""
    out = torch.full((x.shape[1], x.shape[0], x.shape[2] + room), -7, dtype=x.dtype, device=DEV)
    out[..., :x.shape[2]] = x.permute(1, 0, 2).to(DEV)
    return out[..., :x.shape[2]].permute(1, 0, 2)


@pytest.mark.parametrize("seqs,heads", [(3, 2), (1, 4), (5, 1)])
@pytest.mark.parametrize("room", [0, 3])
def test_by_head_as_by_sequence(seqs, heads, room):
    c, lens, _, q = case(BF, 2 * heads, heads, 64, [1] * seqs, [300, 20, 90, 7, 150][:seqs])
    q, L = q.to(DEV), ints(lens)
    lse = torch.zeros(seqs, 2 * heads, device=DEV)
    c.attend(q, L, lse=lse)
    plain = torch.rand(seqs, heads, max(lens), generator=gen(3)).to(DEV)
    other = by_head(plain, room)
    c.weigh(q, L, lse, plain, decay=0.5)
    assert torch.equal(c.weigh(q, L, lse, other, decay=0.5), plain)
    like = dict(dtype=torch.int32)
    kept = [torch.full((seqs, heads, 40), -1, device=DEV, **like), by_head(torch.full((seqs, heads, 40), -1, **like), room)]
    out = [torch.zeros(seqs, heads, 40, device=DEV), by_head(torch.zeros(seqs, heads, 40), room)]
    counts = [c.select(w, L, 40, kept=k, weights_out=o, recent=3)[1] for w, k, o in ((plain, kept[0], out[0]), (other, kept[1], out[1]))]
    assert torch.equal(*kept) and torch.equal(*out) and torch.equal(*counts)
    pool = c.store.pool.clone()
    c.evict(kept[0], counts[0])
    want = c.store.pool.clone()
    c.store.pool.copy_(pool)
    c.evict(kept[1], counts[1])
    assert torch.equal(c.store.pool, want)
    c.select(plain, L, 40, weights_out=plain)
    c.select(other, L, 40, weights_out=other)                                        # in place
    assert torch.equal(plain, other)


def test_rows_that_do_overlap_are_refused():
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1, 1], [9, 9, 9])
    q, lse, L = q.to(DEV), torch.zeros(3, 4, device=DEV), ints(lens)
    room = torch.zeros(1000, device=DEV)
    for seq, head in [(20, 59), (19, 100), (100, 19), (39, 20), (20, 20), (0, 100), (100, 0), (30, 40)]:
        before = c.store.stats()["launches"]
        with pytest.raises(T2IError, match="overlap"):
            c.weigh(q, L, lse, torch.as_strided(room, (3, 2, 20), (seq, head, 1)))
        assert c.store.stats()["launches"] == before
    for seq, head in [(20, 60), (40, 20), (100, 21), (21, 100)]:
        c.weigh(q, L, lse, torch.as_strided(room, (3, 2, 20), (seq, head, 1)))
