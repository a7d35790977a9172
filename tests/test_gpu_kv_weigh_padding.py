"""Accumulated attention of a padded batch (marked gpu): rows behind the last sequence, and those of other sequences, may hold
anything, NaN included, in queries and log-sum-exps; column tiles reach over both."""
import math

import pytest
import torch

from kv_plain import DEV
from test_gpu_kv import BF, HF, case, ints, starts_of
from test_gpu_kv_weigh import sums

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


@pytest.mark.parametrize("dtype,heads,kv", [(BF, 8, 2), (HF, 7, 1), (BF, 160, 1)])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 1, 2], [20, 3, 9], [33, 40, 2], [150, 5, 97]])
@pytest.mark.parametrize("how", ["causal", "window", "spans"])
def test_rows_of_nobody_and_of_others(dtype, heads, kv, new, how):
    c, lens, kvs, q = case(dtype, heads, kv, 64, new, [400, 30, 700])
    pad = 37
    spans = torch.tensor([(5, L - m) for m, L in zip(new, lens) for _ in range(m)] + [(0, 1 << 30)] * pad)
    opt = {"causal": {}, "window": dict(window=60), "spans": {}}[how]
    lse = sums(new, kvs, q, 64, spans=spans if how == "spans" else None, **opt)
    q = torch.cat([q, torch.full((pad, heads, 64), math.nan, dtype=dtype)]).to(DEV)
    lse = torch.cat([lse, torch.full((pad, heads), math.nan)]).to(DEV)
    if how == "spans":
        opt["spans"] = spans.int().to(DEV)
    L, starts = ints(lens), starts_of(new)
    n, edges = sum(new), [0, new[0], new[0] + new[1], sum(new)]

    def weigh(q, lse):
        w = torch.full((3, kv, max(lens)), 0.25, device=DEV)
        return c.weigh(q, L, lse, w, starts=starts, max_new=max(new), decay=0.5, **opt)

    clean = weigh(torch.where(q.isnan(), 0, q), torch.where(lse.isnan(), 0, lse))
    assert torch.equal(weigh(q, lse), clean) and torch.isfinite(clean).all()
    # each sequence alone is clean, the others' rows NaN
    for s in range(3):
        mine = torch.zeros(n + pad, dtype=torch.bool, device=DEV)
        mine[edges[s]:edges[s + 1]] = True
        got = weigh(torch.where(mine[:, None, None], q, math.nan), torch.where(mine[:, None], lse, math.nan))
        assert torch.equal(got[s], clean[s]), s
