"""Argument checks of the 8-bit linear layers' and the drafts' C entry points: they come before any
HIP call (no GPU); and the rules that choose a product's kernel."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_11985_amd import _lib
from tests.test_layers_cpu import BIG, INF, INV, NAN, P, WS


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


QUANTIZE = dict(dtype=0, rows=3, cols=8, x=P, ldx=8, q=P, ldq=8, scales=P, stream=None)
LINEAR = dict(dtype=0, rows=3, n_in=8, n_out=5, x=P, ldx=8, x_scales=None, weight=P, ldw=8,
              w_scales=P, bias=P, act=1, residual=P, ldr=5, y=P, ldy=5, ws=P, ws_bytes=1 << 20,
              stream=None)
VERIFY = dict(kind=0, dtype=0, sequences=3, drafts=2, cols=8, target=P, ldt=8, draft=P, ldd=8,
              inv_t=1.0, drafted=P, uniforms=P, outcomes=P, accepted=P, ws=P, ws_bytes=1 << 20,
              stream=None)

REFUSED = [
    ("vqc_quantize", QUANTIZE, [
        (dict(dtype=3), INV), (dict(rows=-1), INV), (dict(cols=-1), INV), (dict(x=None), INV),
        (dict(q=None), INV), (dict(scales=None), INV), (dict(x=P + 2), INV),
        (dict(scales=P + 2), INV), (dict(ldq=7), INV), (dict(ldx=-8), INV),
        (dict(rows=1 << 41), BIG), (dict(rows=1 << 30, cols=1 << 20, ldq=1 << 20), BIG),
        (dict(ldx=1 << 62), BIG)]),
    ("vqc_linear_quantized", LINEAR, [
        (dict(dtype=9), INV), (dict(act=5), INV), (dict(act=-1), INV), (dict(n_in=-1), INV),
        (dict(x=None), INV), (dict(x=P + 2), INV), (dict(x_scales=P + 2), INV),
        (dict(weight=None), INV), (dict(w_scales=None), INV), (dict(w_scales=P + 1), INV),
        (dict(y=None), INV), (dict(ldy=4), INV), (dict(ldw=-1), INV), (dict(residual=P + 1), INV),
        (dict(bias=P + 2), INV), (dict(rows=1 << 39, n_out=4), BIG), (dict(ws=None), WS),
        (dict(ws=P + 8), WS), (dict(ws_bytes=16), WS)]),
    ("vqc_verify_drafts", VERIFY, [
        (dict(kind=2), INV), (dict(dtype=5), INV), (dict(sequences=-1), INV),
        (dict(drafts=-1), INV), (dict(cols=0), INV), (dict(inv_t=0.0), INV),
        (dict(inv_t=NAN), INV), (dict(inv_t=INF), INV), (dict(kind=1, inv_t=2.0), INV),
        (dict(target=None), INV), (dict(target=P + 2), INV), (dict(draft=P + 2), INV),
        (dict(ldt=-1), INV), (dict(drafted=None), INV), (dict(drafted=P + 4), INV),
        (dict(uniforms=None), INV), (dict(uniforms=P + 4), INV), (dict(outcomes=None), INV),
        (dict(accepted=None), INV), (dict(accepted=P + 4), INV), (dict(cols=10 ** 5, ws=None), WS),
        (dict(cols=10 ** 5, ws=P + 8), WS), (dict(cols=10 ** 5, ws_bytes=16), WS),
        (dict(cols=1 << 40), BIG),
        (dict(sequences=1 << 20, drafts=1 << 20), BIG), (dict(drafts=1 << 40), BIG),
        (dict(ldd=1 << 62), BIG)]),
]


@pytest.mark.parametrize("name,good,change,status",
                         [(n, g, c, s) for n, g, cs in REFUSED for c, s in cs],
                         ids=lambda v: str(v) if isinstance(v, (str, int)) else "-".join(
                             f"{k}={x}" for k, x in v.items()) if len(v) < 5 else "")
def test_refused(lib, name, good, change, status):
    assert getattr(lib, name)(*{**good, **change}.values()) == status
    assert _lib.vqc_last_error()


def test_empty_calls_launch_nothing(lib):
    assert lib.vqc_quantize(*{**QUANTIZE, "rows": 0, "x": None, "q": None}.values()) == 0
    assert lib.vqc_linear_quantized(*{**LINEAR, "rows": 0, "x": None, "y": None}.values()) == 0
    assert lib.vqc_linear_quantized(*{**LINEAR, "n_out": 0, "weight": None,
                                      "w_scales": None}.values()) == 0
    assert lib.vqc_verify_drafts(*{**VERIFY, "sequences": 0, "target": None}.values()) == 0


def test_workspace_sizes(lib):
    bad = ctypes.c_size_t(-1).value
    linear, verify = lib.vqc_linear_quantized_workspace_bytes, lib.vqc_verify_drafts_workspace_bytes
    assert linear(-1, 1, 1, 0) == bad and linear(1, 1, 1, 2) == bad and linear(1, 1, 1, -1) == bad
    assert linear(1 << 40, 1 << 40, 1, 0) == bad
    assert linear(0, 0, 0, 0) == 0 and linear(3, 128, 5, 1) == 0
    assert linear(3, 100, 5, 1) == 512  # rows of 128
    assert linear(3, 100, 5, 0) == 768  # and their steps
    assert verify(3, 1, 1, 1, 1) == bad and verify(0, -1, 1, 1, 1) == bad
    assert verify(0, 1, 1, 0, 1) == bad and verify(0, 1, 1, 1, 2) == bad
    assert verify(0, 1 << 30, 1 << 30, 1 << 30, 1) == bad
    assert verify(0, 0, 4, 9, 1) == 0 and verify(2, 1, 4, 9, 1) == 0  # a workgroup per sequence
    assert 0 < verify(2, 1, 4, 90000, 0) < verify(2, 1, 4, 90000, 1)


# ------------------------------------------------------------------ rules

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("tiles") / "quantized_tiles")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-I",
                           os.path.join(ROOT, "paper_2607_11985_amd", "csrc"),
                           os.path.join(ROOT, "tests", "quantized_tiles.cpp"), "-o", exe])

    def ask(sizes):
        """(how, splits) of each (element, rows, n_in, n_out)."""
        text = "".join(" ".join(map(str, s)) + "\n" for s in sizes)
        out = subprocess.run([exe], input=text, text=True, capture_output=True,
                             check=True).stdout
        assert "wrong" not in out
        return [(w[0], int(w[1])) for w in map(str.split, out.splitlines())]
    return ask


def test_sizes_of_the_gpu_tests_reach_every_kernel(ways):
    from tests import test_gpu_quantized as G
    for element in (2, 4):
        found = set(how for how, _ in ways([(element,) + s for s in G.SIZES]))
        assert {"one", "short", "fused", "few", "64", "128", "256"} <= found
    exact = ways([(1,) + s for s in G.EXACT])
    assert {"few", "64", "128", "256"} <= set(how for how, _ in exact)
    assert {1} < set(splits for how, splits in exact if how in ("64", "128"))
    assert {"64", "128", "256"} <= set(how for how, splits in exact if splits > 1)


def test_long_sums_are_split(ways):
    for rows in (1, 3, 20, 70, 3000):
        for k in (131071, 131072, 140000, 300001, 1 << 22):
            (how, splits), = ways([(1, rows, k, 40)])
            assert how.isdigit() and splits >= -(-k // 131071)


# (bytes of an element, rows, n_in, n_out): us of rows quantised where they are multiplied, and of a
# launch of its own for them
SHORT = {(2, 64, 16, 10): (3.6, 8.1), (2, 2048, 256, 512): (6.9, 8.5), (2, 8192, 64, 512): (10.4, 12.1),
         (2, 8192, 128, 512): (13.7, 12.1), (2, 4096, 128, 1024): (13.8, 11.9),
         (2, 8192, 128, 1024): (23, 18), (2, 256, 512, 512): (6.6, 8.3),
         (2, 1000, 1001, 100): (8.2, 10.8), (2, 8192, 512, 64): (8.6, 11.7),
         (2, 1024, 768, 384): (9.9, 9.6), (2, 256, 1024, 1024): (10.2, 9.7),
         (2, 8192, 1000, 40): (12.1, 16.8), (4, 8192, 64, 512): (10.7, 15.0),
         (4, 8192, 128, 1024): (17, 22), (4, 2048, 512, 512): (9.5, 10.1),
         (4, 4096, 256, 2048): (25.5, 23.6), (4, 1000, 1001, 100): (7.2, 10.7),
         (4, 8192, 1000, 40): (11.3, 16.5), (4, 1024, 768, 384): (9.6, 10.2),
         (4, 1024, 1024, 1024): (17.4, 11.5), (2, 4, 512, 512): (5.9, 4.5),
         (2, 16, 1024, 1024): (9.7, 6.8)}


@pytest.mark.parametrize("size", SHORT, ids=str)
def test_short_rows_take_the_faster_way(ways, size):
    (how, _), = ways([size])
    so, other = SHORT[size]
    assert (how == "short") == (so < other)
