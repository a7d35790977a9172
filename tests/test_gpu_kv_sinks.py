"""Attention in a window with a few first slots that stay visible (marked gpu), against a plain form in 64 bits: where
the sinks lie beside, reach into or cover the window, and where the tiles of both meet."""
import math

import numpy as np
import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_bounded import attend64
from kv_plain import DEV, near_attend, words, write_rows
from test_gpu_kv import BF, HF, case, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def check(c, lens, new, kvs, q, tree=None, slopes=None, **opt):
    n, heads, dim = q.shape
    out = torch.full((n, heads, dim), math.nan, dtype=c.dtype, device=DEV)
    lse = torch.full((n, heads), math.nan, device=DEV)
    how = dict(out=out, lse=lse, layer=c.layers - 1, slopes=None if slopes is None else slopes.to(DEV), starts=starts_of(new),
               max_new=max(new), **opt)
    for _ in range(2):  # the second call finds the workspace as the first one left it
        out.fill_(math.nan), lse.fill_(math.nan)
        if tree is not None:
            c.attend_tree(q.to(DEV), ints(lens), tree.to(DEV), **how)
        else:
            c.attend(q.to(DEV), ints(lens), **how)
    at = 0
    for s, (m, L) in enumerate(zip(new, lens)):
        if m == 0:
            continue
        w = slice(at, at + m)
        want = attend64(q[w], *kvs[s], dim ** -0.5, slopes=slopes, tree=None if tree is None else tree[w], **opt)
        near_attend(out[w], lse[w], *want, c.dtype, f"sequence {s} of {m} new tokens, {L} in all, {opt}")
        at += m


# sinks and window: beside one another, in neighbouring tiles, in one tile, touching, overlapping, of more than a tile
PAIRS = [(1, 1), (4, 100), (128, 50), (129, 300), (260, 7), (600, 200), (5000, 3)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sinks,window", PAIRS)
@pytest.mark.parametrize("heads,kv,dim,new,ctx", [
    (8, 2, 128, [1] * 9, [0, 1, 15, 126, 127, 128, 700, 383, 1500]),        # one token: few queries
    (3, 3, 80, [5, 0, 16, 1], [3, 90, 400, 900]),
    (4, 1, 64, [70, 300, 1], [900, 0, 260]),                                # row by row
    (14, 2, 128, [130, 33], [5, 777])])
def test_sinks(dtype, sinks, window, heads, kv, dim, new, ctx):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx, page=262144, layers=2)
    check(c, lens, new, kvs, q, sinks=sinks, window=window)


@pytest.mark.parametrize("how", ["cap", "bias", "all"])
@pytest.mark.parametrize("new,ctx", [([1, 2, 1], [1, 130, 900]), ([60, 300], [700, 100])])
def test_sinks_with_other_options(how, new, ctx):
    heads = 8
    c, lens, kvs, q = case(BF, heads, 2, 64, new, ctx, qs=4.0)
    opt = dict(softcap=6.0) if how != "bias" else {}
    if how != "cap":
        opt["slopes"] = torch.tensor([2.0 ** (-h - 3) for h in range(heads)])
    check(c, lens, new, kvs, q, sinks=9, window=140, **opt)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv", [(8, 2), (64, 1), (2, 2)])
@pytest.mark.parametrize("sinks,window", [(3, 20), (140, 40), (20, 200)])
def test_sinks_of_drafts(dtype, heads, kv, sinks, window):
    """... also where drafted tokens are sinks themselves."""
    new, ctx = [1, 64, 21, 5, 9], [30, 300, 0, 613, 2]
    c, lens, kvs, q = case(dtype, heads, kv, 64, new, ctx)
    rng = np.random.default_rng(sinks)
    check(c, lens, new, kvs, q, tree=torch.cat([words(m, rng) for m in new]), sinks=sinks, window=window)
    few = [min(m, 6) for m in new]
    c, lens, kvs, q = case(dtype, 4, 2, 64, few, ctx)
    check(c, lens, few, kvs, q, tree=torch.cat([words(m, rng) for m in few]), sinks=sinks, window=window)


@pytest.mark.parametrize("new", [[1, 1], [40, 200]])
def test_slots_between_sinks_and_window_may_hold_anything(new):
    c, lens, kvs, q = case(BF, 4, 2, 128, new, [900, 700])
    for s, (m, L) in enumerate(zip(new, lens)):  # NaN and infinities where no token looks, in the sinks' tile too
        k, v = kvs[s]
        k[5:L - m - 50], v[5:L - m - 50] = math.nan, math.inf
        write_rows(c, s, 0, k.to(DEV), v.to(DEV))
        k[5:L - m - 50], v[5:L - m - 50] = 0, 0
    check(c, lens, new, kvs, q, window=50, sinks=5)


@pytest.mark.parametrize("new,ctx", [([1, 3], [300, 20]), ([150, 40], [60, 300])])
def test_sinks_that_change_nothing(new, ctx):
    """Without a window, or none of them: the same bits as the call without."""
    c, lens, kvs, q = case(HF, 8, 2, 128, new, ctx)
    how = dict(starts=starts_of(new), max_new=max(new))
    q, L = q.to(DEV), ints(lens)
    for window in (0, 70):
        want = c.attend(q, L, window=window, **how)
        assert torch.equal(c.attend(q, L, window=window, sinks=0, **how), want)
        if not window:
            assert torch.equal(c.attend(q, L, sinks=40, **how), want)
            assert torch.equal(c.attend(q, L, sinks=(1 << 32) - 1, **how), want)
        else:  # all are sinks: causal
            near = c.attend(q, L, window=window, sinks=(1 << 32) - 1, **how)
            assert torch.equal(near, c.attend(q, L, **how))


def test_refusals():
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1], [9, 9])
    spans = torch.zeros(2, 2, dtype=torch.int32, device=DEV)
    with pytest.raises(T2IError, match="spans"):
        c.attend(q.to(DEV), ints(lens), spans=spans, sinks=1)
    with pytest.raises(ValueError, match="sinks"):
        c.attend(q.to(DEV), ints(lens), window=1, sinks=-1)
    with pytest.raises(ValueError, match="sinks"):
        c.attend_tree(q.to(DEV), ints(lens), torch.ones(2, dtype=torch.int64, device=DEV), window=1, sinks=1 << 32)
