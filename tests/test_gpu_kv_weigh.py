"""Accumulated attention over the cache (marked gpu), against a plain form in 64 bits, at the sizes, masks and places
where it can go wrong. Every byte of a pool that holds no row of the case is NaN."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2607_26566_gb300 import T2IError
from kv_bounded import attend64, near_weights, weigh64
from kv_plain import DEV, write_rows
from test_gpu_kv import BF, HEADS, HF, case, gen, ints, starts_of

pytestmark = pytest.mark.gpu
PAD = 5  # slots of the weights behind the longest sequence


@pytest.fixture(scope="module", autouse=True)
def _built(lib):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    yield


def sums(new, kvs, q, dim, spans=None, scale=None, **opt):
    """lse of every query, in fp32."""
    out, at = torch.zeros(q.shape[:2]), 0
    for s, m in enumerate(new):
        w, (k, v) = slice(at, at + m), kvs[s]
        if m and spans is not None:
            from kv_plain import attend64 as with_spans
            out[w] = with_spans(q[w], k, v, scale or dim ** -0.5, spans=spans[w], **opt)[1].float()
        elif m:
            out[w] = attend64(q[w], k, v, scale or dim ** -0.5, **opt)[1].float()
        at += m
    return out


def check(c, lens, new, kvs, q, decay=1.0, slopes=None, spans=None, scale=None, max_len=0, each=False, lse=None, held=None, **opt):
    n, heads, dim = q.shape
    if lse is None:
        plain = {k: v for k, v in opt.items()}
        lse = sums(new, kvs, q, dim, spans=spans, scale=scale, slopes=slopes, **plain)
    if held is None:
        held = 3 * torch.rand(len(lens), c.kv_heads, max(lens) + PAD, generator=gen(9))
    weights = held.clone().to(DEV)
    how = dict(layer=c.layers - 1, decay=decay, scale=scale, max_len=max_len, slopes=None if slopes is None else slopes.to(DEV),
               spans=None if spans is None else spans.to(torch.int32).to(DEV), **opt)
    if not each:
        how.update(starts=starts_of(new), max_new=max(new))
    assert c.weigh(q.to(DEV), ints(lens), lse.to(DEV), weights, **how) is weights
    again = held.clone().to(DEV)
    c.weigh(q.to(DEV), ints(lens), lse.to(DEV), again, **how)
    assert torch.equal(again.view(torch.int32), weights.view(torch.int32)), "two calls give the same bits"
    got, at = weights.cpu(), 0
    for s, (m, L) in enumerate(zip(new, lens)):
        # behind the sequence, and where there is nothing new: as it was
        assert torch.equal(got[s, :, L if m else 0:].view(torch.int32), held[s, :, L if m else 0:].view(torch.int32)), f"sequence {s}"
        if m == 0:
            continue
        w = slice(at, at + m)
        want, off = weigh64(q[w], kvs[s][0], lse[w], dim ** -0.5 if scale is None else scale, slopes=slopes,
                            spans=None if spans is None else spans[w], **opt)
        near_weights(got[s, :, :L], held[s, :, :L], want, off, L - m, decay, f"sequence {s} of {m} new tokens, {L} in all")
        at += m
    return got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_one_token(dtype, heads, kv, dim):
    new, ctx = [1] * 11, [0, 1, 15, 16, 126, 127, 128, 700, 383, 255, 256]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    check(c, lens, new, kvs, q, each=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", HEADS + [(160, 1, 64), (260, 2, 16)])
@pytest.mark.parametrize("new,ctx", [([3, 0, 17, 1], [5, 40, 0, 300]), ([129, 64], [0, 200]), ([300], [77]), ([4, 2], [600, 3])])
def test_chunks(dtype, heads, kv, dim, new, ctx):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx, page=262144, layers=2)
    check(c, lens, new, kvs, q)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("queries", [16, 20, 32, 36, 64, 132])
def test_many_ragged_sequences(dtype, heads, kv, dim, queries):
    """Around 16, 32 and 128 queries to a key head; some sequences without a token."""
    most = queries * kv // heads
    new = [most if i % 3 == 0 else i % (most + 1) for i in range(170)]
    ctx = [(i * 37) % 300 for i in range(170)]
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    check(c, lens, new, kvs, q, decay=0.5)


@pytest.mark.parametrize("how", ["cap", "wide cap", "bias", "window", "sinks", "far sinks", "all", "window1"])
@pytest.mark.parametrize("decay", [1.0, 0.75, 0.0])
@pytest.mark.parametrize("new,ctx", [([1, 1, 1], [0, 130, 900]), ([2, 9, 5], [3, 127, 600]), ([200, 40], [350, 0])])
def test_score_options(how, decay, new, ctx):
    heads, kv, dim = 8, 2, 64
    c, lens, kvs, q = case(BF, heads, kv, dim, new, ctx, qs=4.0)
    opt = {}
    if how in ("cap", "all"):
        opt["softcap"] = 5.0
    if how == "wide cap":
        opt["softcap"] = 1e5
    if how in ("bias", "all"):
        opt["slopes"] = torch.tensor([2.0 ** (-h - 1) for h in range(heads)])
    if how in ("window", "sinks", "far sinks", "all"):
        opt["window"] = 100
    if how == "window1":
        opt["window"] = 1
    if how != "window" and "window" in opt:
        opt["sinks"] = 270 if how == "far sinks" else 3
    check(c, lens, new, kvs, q, decay=decay, scale=0.2, **opt)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 128), (3, 3, 80)])
@pytest.mark.parametrize("new,ctx", [([1, 1, 1, 1], [5, 200, 300, 0]), ([70, 0, 20], [0, 30, 260]), ([333], [5])])
@pytest.mark.parametrize("decay", [1.0, 0.0])
def test_spans(dtype, heads, kv, dim, new, ctx, decay):
    c, lens, kvs, q = case(dtype, heads, kv, dim, new, ctx)
    rng = np.random.default_rng(dim)
    spans = []
    for m, L in zip(new, lens):
        for _ in range(m):
            a, b = sorted(rng.integers(0, L + 1, 2).tolist())
            spans.append((a, b) if rng.random() < 0.8 else (0, 0))      # a fifth sees nothing
    check(c, lens, new, kvs, q, spans=torch.tensor(spans), decay=decay)


def test_queries_that_count_nothing():
    """lse of -infinity, and all tokens of a sequence so."""
    new, ctx = [3, 40, 2], [300, 10, 5]
    c, lens, kvs, q = case(BF, 4, 2, 64, new, ctx)
    lse = sums(new, kvs, q, 64)
    lse[1], lse[10, 2], lse[43:] = -math.inf, -math.inf, -math.inf
    check(c, lens, new, kvs, q, lse=lse)


@pytest.mark.parametrize("new", [[1, 1], [40, 200]])
def test_what_no_token_sees_may_be_anything(new):
    """Keys outside the window, values anywhere, weights so far where they do not count."""
    c, lens, kvs, q = case(BF, 4, 2, 128, new, [900, 700])
    for s, (m, L) in enumerate(zip(new, lens)):
        k, v = kvs[s]
        k[5:L - m - 50] = math.nan
        k[5:300] = math.inf
        write_rows(c, s, 0, k.to(DEV), torch.full_like(v, math.nan).to(DEV))
        k[5:L - m - 50] = 0
    held = torch.full((2, 2, max(lens) + PAD), math.nan)
    check(c, lens, new, kvs, q, window=50, sinks=5, decay=0.0, held=held)
    held = torch.rand(2, 2, max(lens) + PAD, generator=gen(1))
    for s, (m, L) in enumerate(zip(new, lens)):
        held[s, :, L - m:L] = math.nan                # of the new tokens
    check(c, lens, new, kvs, q, window=50, sinks=5, held=held)


@pytest.mark.parametrize("new", [[1, 1], [40, 3], [200, 30]])
@pytest.mark.parametrize("max_len", [1, 700, 1 << 30])
def test_a_wrong_max_len_changes_no_result(new, max_len):
    c, lens, kvs, q = case(BF, 8, 2, 64, new, [800, 100])
    # (within the bound of the sum: a split elsewhere adds the same terms up in other groups, and fp32 addition is not
    # associative, so the last bits may differ)
    check(c, lens, new, kvs, q, max_len=max_len)


def test_a_negative_scale_and_none():
    c, lens, kvs, q = case(HF, 4, 2, 64, [2, 60], [100, 30])
    check(c, lens, [2, 60], kvs, q, scale=-0.3)
    n = torch.full((62, 4), 3.0)
    check(c, lens, [2, 60], kvs, q, scale=0.0, lse=n)


def test_strides_a_table_of_chosen_rows_and_fewer_slots():
    c, lens, kvs, q = case(HF, 6, 3, 64, [1, 1, 1, 1], [70, 10, 200, 33])
    pick = [2, 0]
    wide = torch.full((2, 20, 64), math.nan, dtype=HF, device=DEV)
    wide[:, 3:9] = q[pick].to(DEV)
    lse = sums([1] * 4, kvs, q, 64)[pick]
    held = torch.rand(2, 5, 150, generator=gen(2))
    weights = held.clone().to(DEV)
    table = torch.full((2, c.max_pages + 5), -1, dtype=torch.int32, device=DEV)
    table[:, 2:2 + c.max_pages] = c.table[pick]
    part = weights[:, 1:4, 7:137]                     # 130 slots of them
    c.weigh(wide[:, 3:9], ints([lens[i] for i in pick]), lse.to(DEV), part, table=table[:, 2:2 + c.max_pages])
    got = weights.cpu()
    for r, i in enumerate(pick):
        L = min(lens[i], 130)
        want, off = weigh64(q[i:i + 1], kvs[i][0], lse[r:r + 1], 0.125)
        near_weights(got[r, 1:4, 7:7 + L], held[r, 1:4, 7:7 + L], want[:, :L], off[:, :L], lens[i] - 1, 1.0)
        got[r, 1:4, 7:7 + L] = held[r, 1:4, 7:7 + L]
    assert torch.equal(got, held), "nothing else was written"


def test_bounds_that_make_no_sense_touch_nothing():
    c, lens, kvs, q = case(BF, 4, 2, 64, [2, 2], [40, 9])
    weights = torch.full((2, 2, 60), 7.0, device=DEV)
    lse = torch.zeros(4, 4, device=DEV)
    for L in ([1, 0], [-5, 1 << 30], [c.max_pages * c.page_tokens + 1, 1]):
        c.weigh(q.to(DEV), ints(L), lse, weights)
    c.weigh(q.to(DEV), ints(lens), lse, weights, starts=ints([4, 0, -3]), max_new=4)
    assert (weights == 7).all()
    # pages that the pool lacks: keys of zeros
    c.weigh(q.to(DEV), ints(lens), lse, weights, table=torch.full((2, c.max_pages), -1, dtype=torch.int32, device=DEV))
    got = weights.cpu()
    # (4 tokens x heads of a group: 2 heads x the tokens that see a slot, exp(0 - 0) each)
    assert torch.equal(got[0, :, :40], torch.full((2, 40), 7.0 + 4)) and torch.equal(got[0, :, 40:42], torch.tensor([[4.0, 2.0]] * 2))
    assert (got[0, :, 42:] == 7).all()


@pytest.mark.parametrize("new", [[1], [32], [2000]])
def test_a_slot_that_gets_nearly_everything(new):
    """Sums of many small weights beside a large one lose nothing of either: a sink, and 2,000 tokens' rest."""
    c, lens, kvs, q = case(BF, 16, 2, 64, new, [1000], page=1 << 20)
    k = kvs[0][0]
    k[0] = 0
    k[0, :, 0] = 8.0
    q[:, :, 0] = 20.0
    k[1:, :, 0] = 0
    write_rows(c, 0, 0, kvs[0][0].to(DEV), kvs[0][1].to(DEV))
    check(c, lens, new, kvs, q)


def test_of_a_gradient_and_other_refusals():
    c, lens, _, q = case(BF, 4, 2, 64, [1, 1], [9, 9])
    q, L = q.to(DEV), ints(lens)
    lse, w = torch.zeros(2, 4, device=DEV), torch.zeros(2, 2, 20, device=DEV)

    def no(error, match, *a, **k):
        before = c.store.stats()["launches"]
        with pytest.raises(error, match=match):
            c.weigh(*a, **k)
        assert c.store.stats()["launches"] == before

    no(ValueError, "gradient", q, L, lse.clone().requires_grad_(), w)
    no(ValueError, "gradient", q, L, lse, w.clone().requires_grad_())
    no(TypeError, "lse", q, L, None, w)
    no(TypeError, "weights", q, L, lse, None)
    no(TypeError, "dtype", q, L, lse, w.double())
    no(TypeError, "dtype", q.half(), L, lse, w)
    no(ValueError, "lse", q, L, lse[:, :2], w)
    no(ValueError, "weights", q, L, lse, w[:1])
    no(ValueError, "weights", q, L, lse, w[:, :1])
    no(ValueError, "weights", q, L, lse, w.transpose(1, 2).contiguous().transpose(1, 2))
    no(T2IError, "overlap", q, L, lse, w[:1].expand(2, -1, -1))
    no(T2IError, "overlap", q, L, torch.as_strided(w, (2, 4), (4, 1)), w)
    no(T2IError, "n_slots", q, L, lse, w[..., :0])
    no(T2IError, "decay", q, L, lse, w, decay=math.inf)
    no(T2IError, "scale", q, L, lse, w, scale=math.nan)
    no(T2IError, "layer", q, L, lse, w, layer=1)
    no(T2IError, "spans", q, L, lse, w, spans=torch.zeros(2, 2, dtype=torch.int32, device=DEV), window=3)
    no(T2IError, "spans", q, L, lse, w, spans=torch.zeros(2, 2, dtype=torch.int32, device=DEV), sinks=3)
    no(T2IError, "max_new", q, L, lse, w, starts=ints([0, 1, 2]))
    no(ValueError, "sinks", q, L, lse, w, sinks=-1)
    no(T2IError, "q: the stride", q[:1].expand(2, -1, -1), L, lse, w)
    no(T2IError, "q: the stride", torch.as_strided(q, (2, 4, 64), (128, 64, 1)), L, lse, w)
    assert c.weigh(q[:0], L[:0], lse[:0], w[:0]).shape == (0, 2, 20)      # nothing to do
    c.close()
    no2 = pytest.raises(ValueError, match="closed")
    with no2:
        c.weigh(q, L, lse, w)


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 300]])
def test_a_wait_that_runs_out_is_reported_and_harms_nothing(new):
    """The loads are left out on request, so that the bounded waits for them run their second."""
    c, lens, kvs, q = case(BF, 8, 2, 128, new, [3000, 50, 1500])
    lse = sums(new, kvs, q, 128).to(DEV)
    q, L = q.to(DEV), ints(lens)
    how = dict(starts=starts_of(new), max_new=max(new))
    room = torch.full((3, 4, max(lens) + 64), 7.0, device=DEV)
    used = torch.full((64 << 20,), 1, dtype=torch.uint8, device=DEV)  # what the workspace finds: notes that look valid
    torch.cuda.synchronize()
    del used
    c.inject_timeout(1)
    c.weigh(q, L, lse, room[:, 1:3, 32:-32], decay=0.0, **how)
    torch.cuda.synchronize()
    assert (room[:, 0] == 7).all() and (room[:, 3] == 7).all() and (room[..., :32] == 7).all()
    assert all((room[s, 1:3, 32 + n:] == 7).all() for s, n in enumerate(lens))
    w = torch.zeros(3, 2, max(lens), device=DEV)
    with pytest.raises(T2IError, match="CUDA.*weigh.*gave up"):
        c.weigh(q, L, lse, w, **how)
    c.weigh(q, L, lse, w, **how)                                      # reported once
    total = w.double().sum()
    assert abs(float(total) - sum(new) * 8) < 1e-3 * sum(new) * 8      # every query's weights add up to 1


@pytest.mark.parametrize("heads,kv,tokens", [(14, 2, 32), (8, 2, 32), (8, 2, 24), (4, 2, 32), (8, 2, 3), (8, 2, 160)])
def test_many_units_to_a_block(heads, kv, tokens):
    """Runs of many units, over key heads and sequences of one and of two column tiles, and of more; some short."""
    new = [tokens, tokens, max(1, tokens // 3), 1, tokens] * 4
    ctx = [2100, 700, 1500, 900, 1] * 4
    c, lens, kvs, q = case(HF, heads, kv, 128, new, ctx, page=262144)
    check(c, lens, new, kvs, q, decay=0.25)
    check(c, lens, new, kvs, q, window=300, sinks=2)


@pytest.mark.parametrize("stride", [4 * 64 + 8, 4 * 64 + 24, 5 * 64, 4 * 64])
@pytest.mark.parametrize("new", [[1, 1], [20, 3], [150, 40]])
def test_strides_between_tokens(stride, new):
    c, lens, kvs, q = case(BF, 4, 2, 64, new, [300, 70])
    n = sum(new)
    wide = torch.full((n * stride,), math.nan, dtype=BF, device=DEV)
    view = torch.as_strided(wide, (n, 4, 64), (stride, 64, 1))
    view.copy_(q)
    lse = sums(new, kvs, q, 64)
    w = torch.zeros(2, 2, max(lens), device=DEV)
    c.weigh(view, ints(lens), lse.to(DEV), w, starts=starts_of(new), max_new=max(new))
    want = torch.zeros_like(w)
    c.weigh(q.to(DEV), ints(lens), lse.to(DEV), want, starts=starts_of(new), max_new=max(new))
    assert torch.equal(w, want) and float(w.sum()) > n * 3.9


@pytest.mark.parametrize("new,most", [([7, 3], 4), ([200, 90], 60)])
def test_tokens_beyond_max_new_are_not_counted(new, most):
    """As they are not attended; their slots are new ones all the same."""
    c, lens, kvs, q = case(BF, 8, 2, 64, new, [100, 40])
    lse = sums(new, kvs, q, 64)
    held = torch.rand(2, 2, max(lens) + PAD, generator=gen(2))
    w = held.clone().to(DEV)
    c.weigh(q.to(DEV), ints(lens), lse.to(DEV), w, starts=starts_of(new), max_new=most)
    at = 0
    for s, (m, L) in enumerate(zip(new, lens)):
        some = lse[at:at + m].clone()
        some[most:] = -math.inf
        want, off = weigh64(q[at:at + m], kvs[s][0], some, 0.125)
        near_weights(w[s, :, :L].cpu(), held[s, :, :L], want, off, L - m, 1.0)
        at += m


class WeighDesc(C.Structure):
    """t2i_kv_weigh_desc, its batch first."""
    _fields_ = [("table", C.c_void_p), ("table_stride", C.c_uint64), ("lens", C.c_void_p), ("starts", C.c_void_p),
                *[(n, C.c_uint32) for n in ("table_pages", "n_seqs", "n_tokens", "max_new", "layer", "reserved")],
                *[(n, C.c_void_p) for n in ("q", "lse", "weights")],
                *[(n, C.c_uint64) for n in ("q_stride", "seq_stride", "head_stride")],
                ("slopes", C.c_void_p), ("spans", C.c_void_p),
                *[(n, C.c_uint32) for n in ("q_heads", "n_slots", "window", "sinks", "max_len")],
                *[(n, C.c_float) for n in ("scale", "softcap", "decay")],
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


def test_strides_whose_bytes_pass_64_bits_are_refused(lib):
    """From C: (tokens - 1) * stride * 2 bytes, or a table's, are a multiple of 2^64. Nothing is launched."""
    c, lens, _, q = case(BF, 1, 1, 64, [1], [20])
    n = (1 << 25) + 1
    q, L = q.to(DEV), ints(lens)
    lse, w = torch.zeros(n, 1, device=DEV), torch.zeros(1, 1, 64, device=DEV)
    room = torch.zeros(1 << 30, dtype=torch.uint8, device=DEV)
    d = WeighDesc(table=c.table.data_ptr(), table_stride=c.max_pages, lens=L.data_ptr(), table_pages=c.max_pages, n_seqs=1, n_tokens=n,
                  q=q.data_ptr(), lse=lse.data_ptr(), weights=w.data_ptr(), q_stride=1 << 38, seq_stride=64, head_stride=64, q_heads=1,
                  n_slots=64, scale=0.125, decay=1.0, workspace=room.data_ptr(), workspace_bytes=room.numel())
    before = c.store.stats()["launches"]
    assert lib.t2i_kv_weigh(c._h, C.byref(d), None) == 1 and "q:" in c.store.last_error()
    many = 1 << 24
    lens_of = torch.zeros(many + 1, dtype=torch.int32, device=DEV)
    d.n_tokens = d.n_seqs = many + 1
    d.lens, d.table_stride, d.q_stride = lens_of.data_ptr(), 1 << 38, 64
    assert lib.t2i_kv_weigh(c._h, C.byref(d), None) == 1 and "table" in c.store.last_error()
    torch.cuda.synchronize()
    assert c.store.stats()["launches"] == before


@pytest.mark.parametrize("heads,kv,tokens", [(4, 4, 1), (8, 2, 7), (8, 2, 14), (8, 2, 24), (14, 2, 32), (8, 2, 160)])
def test_units_that_no_token_sees_between_others(heads, kv, tokens):
    """A window in sequences of many units, and weights that decay everywhere: most units have nothing to add up, in each
    of the forms (one column tile of 16 to 128 columns, two, many), some of them the first or the last of a block."""
    new = [tokens, 1, tokens, max(1, tokens // 2)] * 5
    ctx = [2500, 1300, 700, 2000] * 5
    c, lens, kvs, q = case(BF, heads, kv, 64, new, ctx, page=262144)
    check(c, lens, new, kvs, q, decay=0.5, window=200, sinks=3)
    check(c, lens, new, kvs, q, decay=0.0, window=200, sinks=700)


@pytest.mark.parametrize("heads,kv,dim,new,ctx", [(8, 2, 64, [40, 33], [700, 1500]), (8, 2, 128, [24, 31, 2], [600, 90, 800]),
                                                  (4, 4, 64, [12, 1], [900, 300])])
@pytest.mark.parametrize("bias", [False, True])
def test_spans_of_long_contexts(heads, kv, dim, new, ctx, bias):
    """Two column tiles, one of 128 and one of 16 columns; far units that no token sees."""
    c, lens, kvs, q = case(HF, heads, kv, dim, new, ctx)
    rng = np.random.default_rng(dim)
    spans = []
    for m, L in zip(new, lens):
        for i in range(m):
            a = int(rng.integers(0, 300)) if i % 3 else L - m
            spans.append((a, min(L, a + int(rng.integers(1, 200)))) if i % 5 else (0, 0))
    opt = dict(slopes=torch.tensor([2.0 ** (-h - 4) for h in range(heads)]), softcap=30.0) if bias else {}
    check(c, lens, new, kvs, q, spans=torch.tensor(spans), decay=0.5, **opt)
