"""The key/value cache on the CPU: page geometry and its refusals, and the order
that a hold gives (csrc/deps.hpp against a recording CUDA runtime)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2607_26566_gb300 import _lib as L
from paper_2607_26566_gb300 import build as b
from test_deps import DRIVER, FAKE_RUNTIME


@pytest.mark.parametrize("page,layers,heads,dim,want", [
    (65536, 1, 8, 128, 16), (2 << 20, 28, 8, 128, 16), (65536, 1, 16, 80, 8), (65536, 1, 3, 128, 32), (256, 1, 1, 8, 8),
    (1 << 30, 1, 1, 8, 1 << 25), (65536, 2, 2, 64, 64)])
def test_page_tokens_is_the_largest_power_of_two_that_fits(lib, page, layers, heads, dim, want):
    out = C.c_uint32()
    lay = L.KvLayout(layers, heads, dim, L.BF16)
    assert lib.t2i_kv_page_tokens(page, C.byref(lay), C.byref(out)) == L.OK
    assert out.value == want
    row = layers * heads * dim * 4
    assert want * row <= page < 2 * want * row


@pytest.mark.parametrize("page,lay,why", [
    (65536, (1, 8, 132, 0), "head_dim"), (65536, (1, 8, 136, 0), "head_dim"), (65536, (1, 8, 0, 0), "head_dim"),
    (65536, (1, 0, 64, 0), "kv_heads"), (65536, (0, 8, 64, 0), "layers"), (65536, (1, 8, 64, 2), "dtype"),
    (65536, (2, 64, 128, 0), "8 tokens"), (256, (1, 1, 16, 1), "8 tokens"), (1 << 20, (1, 1 << 31, 64, 0), "kv_heads"),
    (1 << 20, (1 << 31, 1, 64, 0), "layers")])
def test_layouts_that_are_refused(lib, page, lay, why):
    out = C.c_uint32(7)
    k = L.KvLayout(*lay)
    assert lib.t2i_kv_page_tokens(page, C.byref(k), C.byref(out)) == L.ERR_INVALID
    assert out.value == 0 and why in lib.t2i_last_error(None).decode()


def test_null_arguments(lib):
    h = C.c_void_p(5)
    k = L.KvLayout(1, 1, 64, 0)
    assert lib.t2i_kv_page_tokens(65536, None, C.byref(C.c_uint32())) == L.ERR_INVALID
    assert lib.t2i_kv_create(None, C.byref(k), C.byref(h)) == L.ERR_INVALID and not h.value
    assert lib.t2i_kv_create(None, C.byref(k), None) == L.ERR_INVALID
    assert lib.t2i_kv_destroy(None) == L.OK
    for call in (lib.t2i_kv_append, lib.t2i_kv_attend, lib.t2i_kv_commit):
        assert call(None, None, None) == L.ERR_INVALID
    assert lib.t2i_hold(None, None, 1, None) == L.ERR_INVALID


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    """test_deps.py's driver with one more verb, h(old)."""
    d = tmp_path_factory.mktemp("hold")
    (d / "cuda_runtime.h").write_text(FAKE_RUNTIME)
    text = DRIVER.replace("if (verb == 'p') d.writes(0);", "if (verb == 'p' || verb == 'h') d.writes(0);")
    text = text.replace("if (verb == 'v') {", "if (verb == 'h') { d.mark_hold(0); return; }\n        if (verb == 'v') {")
    assert text.count("'h'") == 2
    (d / "main.cpp").write_text(text)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-I", str(d), "-I", b.CSRC, str(d / "main.cpp"),
                    "-o", str(d / "deps")], check=True)
    return str(d / "deps")


@pytest.mark.parametrize("calls,want", [
    ("hA kA kA gB", [2, 0, 0]),              # a read waits for all the holder was given
    ("hA kA pB", [1, 0, 0]),                 # so does a put that reuses the page
    ("gC pA kA hB", [1, 0, 0]),              # a hold waits for the page's writer (the call, not what came after it)
    ("pA gB gC kC hD", [1, 1, 1]),           # ... and its readers
    ("vA kA kA hB", [2, 0, 0]),              # ... and views, which last
    ("hA kA gB kA pC", [2, 1, 0]),           # the hold goes on behind another stream's read
    ("hA kA hB kA kB pC", [0, 1, 0]),        # held for B: B's work, which is behind A's up to then
    ("hA kA hB gC", [0, 0, 0]),              # B has no work yet; A's is behind B's event
    ("hA kA gB kB hA", [0, 1, 0]),           # held again: after B's read
    ("hA kA gA gB", [2, 0, 0]),              # calls of the store on the holder's stream end nothing
    ("hA kA gA kA pB", [3, 0, 0]),
])
def test_a_hold_orders_the_pages_users(driver, calls, want):
    out = subprocess.run([driver, *calls.split()], capture_output=True, text=True, check=True).stdout
    got = [int(x) for x in out.split()]
    assert got == want


def test_destroy_waits_for_a_holder(driver):
    out = subprocess.run([driver, *"hA kA gB kA x".split()], capture_output=True, text=True, check=True).stdout
    assert [int(x) for x in out.split()] == [2, 1, 0]
