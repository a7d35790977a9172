"""The calls that keep a cache bounded, on the CPU: null arguments, the header's structs from C, and the plain forms
against one another."""
import ctypes as C
import itertools
import math
import subprocess

import pytest
import torch

from paper_2607_26566_gb300 import _lib as L
from paper_2607_26566_gb300 import build as b
from kv_bounded import attend64, select_plain, weigh64


def test_null_arguments(lib):
    for call in (lib.t2i_kv_weigh, lib.t2i_kv_select, lib.t2i_kv_evict):
        assert call(None, None, None) == L.ERR_INVALID
    assert lib.t2i_kv_weigh_workspace_bytes(None, 1, 1, C.byref(C.c_uint64())) == L.ERR_INVALID


def test_the_descriptors_are_plain_c(tmp_path):
    src = tmp_path / "d.c"
    src.write_text('#include "t2istore.h"\n#include <stddef.h>\n'
                   "_Static_assert(offsetof(t2i_kv_attend_desc, sinks) == offsetof(t2i_kv_attend_desc, softcap) + 4, \"\");\n"
                   "int f(t2i_kv* k, void* s) {\n"
                   "  t2i_kv_weigh_desc w = {0}; t2i_kv_select_desc c = {0}; t2i_kv_evict_desc e = {0};\n"
                   "  w.decay = 1.0f; c.keep = 1; e.layers = 1;\n"
                   "  return t2i_kv_weigh(k, &w, s) | t2i_kv_select(k, &c, s) | t2i_kv_evict(k, &e, s);\n}\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-c", str(src), "-I" + b.INCLUDE, "-o", str(tmp_path / "d.o")], check=True)


def test_the_plain_choice_is_the_best_of_all():
    """Against every choice of a short row: the sum of what stays is the largest, of equals the first slots."""
    w = [0.0, 3.0, 1.0, 1.0, -0.0, 2.0, 1.0, 0.0]
    for n, a, r in itertools.product(range(9), range(4), range(4)):
        s, t = min(a, n), min(r, n - min(a, n))
        fixed = list(range(s)) + list(range(8 - t, 8))
        rest = [j for j in range(s, 8 - t)]
        best = max(itertools.combinations(rest, n - s - t), key=lambda c: (sum(w[j] for j in c), [-j for j in c]))
        assert select_plain(w, n, a, r) == sorted(fixed + list(best))
    assert select_plain([math.nan, -math.inf, 5.0, math.nan], 2, 0, 0) == [1, 2]
    assert select_plain([math.nan, -math.inf, 5.0, math.nan], 3, 0, 0) == [0, 1, 2]


@pytest.mark.parametrize("window,sinks", [(0, 0), (4, 0), (4, 2), (1, 3)])
def test_the_plain_weights_add_up_to_one_a_query(window, sinks):
    g = torch.Generator().manual_seed(0)
    q, key = torch.randn(5, 4, 8, generator=g), torch.randn(11, 2, 8, generator=g)
    lse = attend64(q, key, key, 0.3, window=window, sinks=sinks)[1].float()
    got, off = weigh64(q, key, lse, 0.3, window=window, sinks=sinks)
    assert abs(float(got.sum()) - 20) < 1e-4 and (off >= 0).all()
    if window:
        hidden = torch.ones(11, dtype=torch.bool)
        hidden[max(0, 6 - window + 1):] = False
        hidden[:sinks] = False
        assert (got[:, hidden] == 0).all()
