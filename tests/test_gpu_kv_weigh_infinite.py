"""Accumulated attention over keys with infinities (marked gpu): a slot whose scores are all -infinity gets nothing, in each
form of the kernel, with columns of a tile that no query has (a tile's columns are 16, 32, 64 or 128)."""
import math

import pytest
import torch

from kv_bounded import attend64, near_weights, scores64, visible
from kv_plain import DEV, write_rows
from test_gpu_kv import BF, HF, case, gen, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def weigh64(q, key, lse, scale, **opt):
    """As kv_bounded's, with a bound from the scores that are finite: an infinite one has no rounding, its weight is 0."""
    m, H, _ = q.shape
    L, K = key.shape[0], key.shape[1]
    see, pos, kpos = visible(m, L, opt.get("window", 0))
    got, off = torch.zeros(K, L, dtype=torch.float64), torch.zeros(K, L, dtype=torch.float64)
    for h in range(H):
        x, _ = scores64(q, key, h, see, pos, kpos, scale, opt.get("softcap", 0.0), opt.get("slopes"))
        raw = q[:, h].double() @ key[:, h // (H // K)].double().T * scale
        big = raw.masked_fill(~see | raw.isinf(), 0).abs().amax(-1)
        p = torch.exp(x - lse[:, h].double()[:, None])
        got[h // (H // K)] += p.sum(0)
        off[h // (H // K)] += ((1e-5 + 2.0 ** -20 * big)[:, None] * p).sum(0) + m * 2.0 ** -126
    return got, 1.01 * off


# queries to a key head: 4, 7, 16, 20, 36, 80, 119 (one tile of 16 to 128 columns), 2 x 68, 2 x 119, 10 x 120, 12 x 119, 2 x 96
FORMS = [(8, 2, [1, 1]), (7, 1, [1, 1]), (8, 2, [4, 1]), (8, 2, [5, 2]), (8, 2, [9, 1]), (8, 2, [20, 7]), (7, 1, [17, 3]),
         (8, 2, [34, 5]), (7, 1, [34, 20]), (8, 2, [300, 60]), (7, 1, [204, 9]), (96, 1, [2, 1])]


@pytest.mark.parametrize("dtype,dim,how", [(BF, 128, "plain"), (HF, 80, "plain"), (BF, 64, "plain"), (HF, 8, "plain"),
                                           (BF, 64, "bias"), (HF, 128, "cap"), (BF, 128, "window")])
@pytest.mark.parametrize("heads,kv,new", FORMS)
def test_slots_whose_scores_are_all_minus_infinity(dtype, dim, heads, kv, new, how):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, [700, 300])
    q[..., 0] = q[..., 0].abs() + 0.5                       # (0 times an infinity is no number, in the formula too)
    opt = {"plain": {}, "bias": dict(slopes=torch.tensor([2.0 ** -(h % 8 + 4) for h in range(heads)])), "cap": dict(softcap=6.0),
           "window": dict(window=150)}[how]
    lse, want, at = torch.zeros(q.shape[:2]), [], 0
    for s, (m, L) in enumerate(zip(new, lens)):
        k, v = kvs[s]
        k[1:L:3, :, 0] = -math.inf
        write_rows(c, s, 0, k.to(DEV), v.to(DEV))
        w = slice(at, at + m)
        lse[w] = attend64(q[w], k, v, dim ** -0.5, **opt)[1].float()
        want.append(weigh64(q[w], k, lse[w], dim ** -0.5, **opt))
        at += m
    held = torch.rand(2, kv, max(lens), generator=gen(5))
    weights = held.clone().to(DEV)
    c.weigh(q.to(DEV), ints(lens), lse.to(DEV), weights, starts=starts_of(new), max_new=max(new), decay=0.5,
            **{k: v.to(DEV) if torch.is_tensor(v) else v for k, v in opt.items()})
    for s, (m, L) in enumerate(zip(new, lens)):
        near_weights(weights[s, :, :L].cpu(), held[s, :, :L], *want[s], L - m, 0.5, f"sequence {s}")
