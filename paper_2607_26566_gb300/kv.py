"""A key/value cache in a store's pages (t2i_kv_*): binding and page upkeep.

:class:`KVCache` reserves pages of a :class:`Store` for the sequences of a text
model and keeps their page table on the device; its calls append keys and
values to the pages, attend over them in place and keep those that got most
attention. As in the rest of the binding, arguments are only marshalled here: the kernels are the library's.
"""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from . import _lib as L
from .store import Store, T2IError, put_descs

L.load()
try:
    from . import _kvcall as _kv
except ImportError as e:
    raise ImportError("the key/value cache's binding is not built: run `python -m paper_2607_26566_gb300.build`") from e

_DTYPES = {torch.bfloat16: L.BF16, torch.float16: L.F16, torch.float32: L.F32}


def page_tokens(page_bytes: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, layers: int = 1) -> int:
    """Tokens of a page (t2i_kv_page_tokens): the largest power of two that fits."""
    lib = L.load()
    out = C.c_uint32()
    lay = L.KvLayout(layers, kv_heads, head_dim, _dtype(dtype))
    st = lib.t2i_kv_page_tokens(page_bytes, C.byref(lay), C.byref(out))
    if st != L.OK:
        raise T2IError(st, lib.t2i_last_error(None).decode())
    return int(out.value)


def _dtype(dt) -> int:
    try:
        return _DTYPES[dt]
    except KeyError:
        raise TypeError(f"the cache has no {dt}") from None


class KVCache:
    """Keys and values of up to ``max_seqs`` sequences of up to ``max_tokens``
    tokens, in pages of ``store``.

    A page holds ``page_tokens`` tokens of one sequence, all ``layers`` of them
    (a model whose layers do not fit one page takes several caches).
    ``table`` is the page table: int32 [max_seqs, max_pages] on the store's
    device, -1 where a sequence has no page. :meth:`reserve` and
    :meth:`release` change it; after a compaction of the store call
    :meth:`refresh`. The pages belong to the stream they were last reserved,
    refreshed or held for (:meth:`hold`): calls on other streams,
    :meth:`release` among them, need a ``hold`` first. ``stream``: a stream or
    its address (0: the default one), None for the device's current one; an
    output that a call makes belongs to the call's stream, like a tensor made
    on it.

    The calls take the first rows of the table, one a sequence, unless
    ``table`` names others (``cache.table[slots]``). Token arrays are
    [tokens, heads, head_dim], the heads of a token next to one another, any
    stride between tokens that is a multiple of 8 (of one token any). ``lens`` is the number of
    each sequence's tokens with the new ones (int32), ``starts`` the first new
    token of each and the end (int32), without it every sequence has as many;
    ``max_new`` goes with it: the most new tokens of a sequence.

    The calls have no gradients: a tensor that requires one is refused unless
    gradients are off (``torch.no_grad()``).

    An attention's workspace comes from torch's allocator for the time of the
    call. Calls that ``torch.cuda.graph`` captures have the graph's memory; a
    capture by other means takes the C call, with a workspace that it keeps."""

    def __init__(self, store: Store, kv_heads: int, head_dim: int, dtype=torch.bfloat16, layers: int = 1,
                 max_seqs: int = 1, max_tokens: int = 4096, stream=None):
        self._lib = L.load()
        self.store, self.dtype = store, dtype
        self.layers, self.kv_heads, self.head_dim = int(layers), int(kv_heads), int(head_dim)
        self._scale = self.head_dim ** -0.5
        self.page_tokens = page_tokens(store.page_bytes, kv_heads, head_dim, dtype, layers)
        self.max_seqs = int(max_seqs)
        self.max_pages = max(1, -(-int(max_tokens) // self.page_tokens))
        self.device = torch.device("cuda", store.device)
        self._host = np.full((self.max_seqs, self.max_pages), -1, np.int32)
        self._ids = [[] for _ in range(self.max_seqs)]     # the objects of each sequence, in token order
        self._pages = [0] * self.max_seqs                  # pages of each sequence
        s = self._stream(stream)
        with torch.cuda.stream(s):
            self.table = torch.full((self.max_seqs, self.max_pages), -1, dtype=torch.int32, device=self.device)
        s.synchronize()  # whichever stream writes or reads it next
        # the handle last: a cache that could not be made leaves none behind
        lay = L.KvLayout(self.layers, self.kv_heads, self.head_dim, _dtype(dtype))
        h = C.c_void_p()
        st = self._lib.t2i_kv_create(store._h, C.byref(lay), C.byref(h))
        if st != L.OK:
            raise T2IError(st, self._lib.t2i_last_error(None).decode())
        try:
            self._c = _kv.cache(int(h.value), store.device, _dtype(dtype), self.kv_heads, self.head_dim, self.table)
        except BaseException:
            self._lib.t2i_kv_destroy(h)
            raise
        self._h = h
        store._users.add(self)

    def close(self):
        """Frees the pages of every sequence and the handle; later calls are
        refused. Closing the store closes its caches."""
        if getattr(self, "_h", None):
            if self.store._h:
                ids = [i for s in self._ids for i in s]
                if ids:
                    self.store.free(np.array(ids, np.uint64))
            _kv.close(self._c)
            self._lib.t2i_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:  # the interpreter is going down
            pass

    def _stream(self, stream):
        """The torch stream that a ``stream`` argument names, as the library's calls take it: None is the device's
        current one, a number a stream's address (0: the default one)."""
        if stream is None:
            return torch.cuda.current_stream(self.device)
        if isinstance(stream, torch.cuda.Stream):
            return stream
        at = int(stream) if isinstance(stream, int) else int(stream.cuda_stream)
        return torch.cuda.ExternalStream(at, device=self.device) if at else torch.cuda.default_stream(self.device)

    def _open(self):
        if not getattr(self, "_h", None):
            raise ValueError("the cache is closed")

    # ---------------------------------------------------------------- pages
    def reserve(self, tokens, seqs=None, stream=None):
        """Pages for sequence ``seqs[i]`` (default: i) to hold ``tokens[i]``
        tokens; sequences that hold as many already keep theirs. All or
        nothing: T2IError (NOSPACE) where the store has no room."""
        self._open()
        seqs = range(len(tokens)) if seqs is None else [int(s) for s in seqs]
        if len(seqs) != len(tokens) or len(set(seqs)) != len(seqs):
            raise ValueError("one number of tokens for each sequence, each named once")
        grow = []
        for s, n in zip(seqs, tokens):
            need = -(-int(n) // self.page_tokens)
            if not 0 <= s < self.max_seqs or need > self.max_pages:
                raise ValueError(f"sequence {s} of {int(n)} tokens is outside the cache "
                                 f"({self.max_seqs} sequences of {self.max_pages * self.page_tokens} tokens)")
            if need > self._pages[s]:
                grow.append((s, need - self._pages[s]))
        if not grow:
            return
        stream = self._stream(stream)
        nbytes = np.array([k for _, k in grow], np.uint64) * np.uint64(self.store.page_bytes)
        st, ids = self.store.put_batch(put_descs(np.zeros(len(grow), np.uint64), nbytes=nbytes), stream)
        self.store.check(st)
        st = self.store.hold(ids, stream)
        if st != L.OK:
            message = self.store.last_error()
            self.store.free(ids)
            raise T2IError(st, message)
        for (s, k), i in zip(grow, ids):
            self._host[s, self._pages[s]:self._pages[s] + k] = self.store.ctl.object(int(i))[2]
            self._pages[s] += k
            self._ids[s].append(int(i))
        self._upload([s for s, _ in grow], stream)

    def release(self, seqs, stream=None):
        """Gives the pages of these sequences back to the store."""
        self._open()
        seqs = list(dict.fromkeys(int(s) for s in seqs))
        for s in seqs:
            if not 0 <= s < self.max_seqs:
                raise ValueError(f"sequence {s} is outside the cache ({self.max_seqs} sequences)")
        ids = [i for s in seqs for i in self._ids[s]]
        if not ids:
            return
        self.store.check(self.store.free(np.array(ids, np.uint64)))
        for s in seqs:
            self._ids[s], self._pages[s] = [], 0
            self._host[s] = -1
        self._upload(seqs, stream)

    def refresh(self, stream=None):
        """After a compaction of the store: the pages' new places."""
        self.hold(stream)
        for s in range(self.max_seqs):
            pages = [p for i in self._ids[s] for p in self.store.ctl.object(i)[2]]
            self._host[s, :len(pages)] = pages
        self._upload(range(self.max_seqs), stream)

    def hold(self, stream=None):
        """Gives the pages to ``stream``, after all that the stream that had
        them was given so far."""
        self._open()
        self.store.check(self.store.hold(np.array([i for s in self._ids for i in s], np.uint64), self._stream(stream)))

    def pages(self, seq: int) -> list:
        """The page numbers of a sequence, in token order."""
        return self._host[seq, :self._pages[seq]].tolist()

    def _upload(self, seqs, stream):
        lo, hi = min(seqs), max(seqs) + 1
        with torch.cuda.stream(self._stream(stream)):
            self.table[lo:hi].copy_(torch.from_numpy(self._host[lo:hi].copy()))

    # ---------------------------------------------------------------- calls
    def _output(self, q, stream):
        # (of the stream that writes it: torch's allocator goes by the stream that a block was made on)
        if stream is None:
            return torch.empty(q.shape, dtype=self.dtype, device=self.device)
        with torch.cuda.stream(self._stream(stream)):
            return torch.empty(q.shape, dtype=self.dtype, device=self.device)

    def _done(self, st):
        raise T2IError(st, self.store.last_error())

    def append(self, k, v, lens, q=None, q_out=None, starts=None, max_new=0, layer=0, q_norm=None, k_norm=None, eps=1e-6,
               cos=None, sin=None, interleaved=False, positions=None, table=None, stream=None):
        """Keys and values of new tokens to their slots (t2i_kv_append).

        ``q``, ``k``, ``v``: of one type, bf16, fp16 or fp32. ``q_out``: of the
        cache's type; may be ``q`` itself. ``q_norm`` / ``k_norm``: fp32
        [head_dim] weights of an RMS norm over each head. ``cos`` / ``sin``: fp32
        [positions, rotary_dim / 2]; the first ``rotary_dim`` elements of a head
        turn, as pairs (i, i + rotary_dim / 2) or, ``interleaved``, (2i, 2i + 1).
        ``positions``: int32 [tokens], a token's slot by default. In fp32, rounded
        once. Returns ``q_out`` (made where only ``q`` is given)."""
        if q_out is None and q is not None:
            q_out = self._output(q, stream)
        st = _kv.append(self._c, k, v, lens, q, q_out, starts, max_new, layer, q_norm, k_norm, eps, cos, sin, interleaved,
                        positions, table, stream)
        if st:
            self._done(st)
        return q_out

    def attend(self, q, lens, out=None, lse=None, starts=None, max_new=0, layer=0, scale=None, softcap=0.0, slopes=None,
               window=0, spans=None, max_len=0, table=None, stream=None, sinks=0):
        """Attention of new tokens over the cache (t2i_kv_attend). Returns ``out``.

        ``scale``: 1 / sqrt(head_dim) by default. ``softcap``: scores become
        softcap * tanh(score / softcap). ``slopes``: fp32 [heads], less slope *
        distance. ``window``: a token sees the last ``window`` slots up to its own.
        ``sinks``: beside a window, and the first ``sinks`` slots (up to its own).
        ``spans``: int32 [tokens, 2], the slots [first, last) that a token sees
        instead (documents, prefixes, padding: an empty one gives zeros).
        ``lse``: fp32 [tokens, heads], receives log(sum(exp(scores))).
        ``max_len``: the longest of ``lens``, where the caller knows it (it only
        sets how the work is split)."""
        if out is None:
            out = self._output(q, stream)
        st = _kv.attend(self._c, q, lens, out, lse, starts, max_new, layer, self._scale if scale is None else scale, softcap,
                        slopes, window, spans, None, max_len, table, stream, sinks)
        if st:
            self._done(st)
        return out

    def attend_tree(self, q, lens, tree, out=None, lse=None, starts=None, max_new=0, layer=0, scale=None, softcap=0.0,
                    slopes=None, window=0, max_len=0, table=None, stream=None, sinks=0):
        """:meth:`attend` for drafted tokens, at most 64 a sequence, the last ones
        of its ``lens``. ``tree``: int64 [tokens], bit i of a token's word is set
        where it sees drafted token i of its sequence (its ancestors and itself);
        it sees all that came before the draft. A drafted token's position, for a
        window, sinks or slopes, is the draft's first slot + the number of its ancestors."""
        if tree is None:
            raise TypeError("tree must be a tensor")
        if out is None:
            out = self._output(q, stream)
        st = _kv.attend(self._c, q, lens, out, lse, starts, max_new, layer, self._scale if scale is None else scale, softcap,
                        slopes, window, None, tree, max_len, table, stream, sinks)
        if st:
            self._done(st)
        return out

    def commit(self, ctx, path, counts, table=None, stream=None):
        """Keeps the accepted tokens of a draft (t2i_kv_commit): in every layer,
        the rows of slot ctx[s] + path[s, i] move to slot ctx[s] + i, i <
        counts[s]. ``path``: int32 [sequences, any], ascending."""
        st = _kv.commit(self._c, ctx, path, counts, table, stream)
        if st:
            self._done(st)

    # -------------------------------------------------------- a cache that stays bounded
    def weigh(self, q, lens, lse, weights, starts=None, max_new=0, layer=0, scale=None, softcap=0.0, slopes=None, window=0,
              sinks=0, spans=None, decay=1.0, max_len=0, table=None, stream=None):
        """Adds the attention that slots got from new tokens to ``weights``
        (t2i_kv_weigh), which it returns: fp32 [sequences, kv_heads, slots].

        For a slot, the sum of exp(score - lse) over the new tokens that see it
        and the heads that share its key head; ``q``, ``lse`` and the options
        are those of the :meth:`attend` before it (``q``'s tokens lie apart). A slot that was there before
        has ``decay`` times what it had added (0: nothing, whatever that was);
        the new tokens' slots start with their sum, slots behind them are left as
        they are. The last tokens of a prompt alone, as new tokens, give what an
        observation window sees. ``weights`` shares no memory with what the call
        reads; its heads may lie inside its sequences or around them. A prompt's
        chunk and other sequences' single tokens go faster as two calls."""
        st = _kv.weigh(self._c, q, lens, lse, weights, starts, max_new, layer, self._scale if scale is None else scale, softcap,
                       slopes, window, sinks, spans, decay, max_len, table, stream)
        if st:
            self._done(st)
        return weights

    def select(self, weights, lens, keep, kept=None, counts=None, weights_out=None, recent=0, sinks=0, keeps=None, max_len=0,
               stream=None):
        """Which slots stay (t2i_kv_select): of each sequence and head of
        ``weights`` (fp32 [sequences, heads, slots]) at most ``keep``: the first
        ``sinks``, the last ``recent`` and those of largest weight (of equals the
        first). ``keeps``: int32 [sequences], fewer of some. ``weights_out``:
        receives the weights of what stays, in order; may be ``weights`` itself.

        Returns ``kept``, int32 [sequences, heads, ...], the slots in ascending
        order (what lies behind their number is left as it is), and ``counts``,
        int32 [sequences], their number: the new ``lens``."""
        if (kept is None or counts is None) and torch.is_tensor(weights) and weights.dim() == 3:  # (others are refused below)
            with torch.cuda.stream(self._stream(stream)):
                if kept is None:
                    kept = torch.empty((*weights.shape[:2], max(0, min(int(keep), weights.shape[2]))), dtype=torch.int32,
                                       device=self.device)
                if counts is None:
                    counts = torch.empty(weights.shape[0], dtype=torch.int32, device=self.device)
        st = _kv.select(self._c, weights, lens, keep, keeps, kept, counts, weights_out, recent, sinks, max_len, stream)
        if st:
            self._done(st)
        return kept, counts

    def evict(self, kept, counts, layer=None, table=None, stream=None):
        """Moves the rows of the slots that stay together (t2i_kv_evict): for each
        key head, of slot kept[s, head, i] to slot i, i < counts[s], in ``layer``,
        or in all of them. ``kept``: int32 [sequences, kv_heads, any], ascending
        (one list for all heads: ``kept.expand(-1, kv_heads, -1)``). The sequence
        then has counts[s] tokens; a token's position is not its slot any more
        (``append`` takes ``positions``). Pages behind them stay with the sequence."""
        st = _kv.evict(self._c, kept, counts, 0 if layer is None else layer, self.layers if layer is None else 1, table, stream)
        if st:
            self._done(st)

    def inject_timeout(self, countdown: int):
        """t2i_kv_inject_timeout (testing)."""
        self._open()
        self._lib.t2i_kv_inject_timeout(self._h, countdown)
