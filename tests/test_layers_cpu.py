"""Argument checks of the layers' C entry points: they come before any HIP call (no GPU)."""
import ctypes
import re

import pytest

from paper_2607_11985_amd import _lib

P = 0x1000  # an aligned address that is never read: every call here is refused or empty
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_header_constants():
    defs = dict(re.findall(r"#define\s+(VQC_\w+)\s+(-?\d+)", open(_lib.HEADER).read()))
    assert [int(defs[k]) for k in ("VQC_F32", "VQC_F16", "VQC_BF16")] == \
        [_lib.DTYPE[k] for k in ("float32", "float16", "bfloat16")]
    for k, v in _lib.ACT.items():
        assert int(defs["VQC_ACT_" + k.upper()]) == v
    for k, v in _lib.SCORES.items():
        assert int(defs["VQC_SCORES_" + k.upper()]) == v
    assert int(defs["VQC_MAX_TOP"]) == _lib.VQC_MAX_TOP


NORM = dict(dtype=0, rows=3, cols=8, x=P, ldx=8, weight=P, bias=P, eps=1e-5, y=P, ldy=8, mean=P,
            rstd=P, stream=None)
NORM_B = dict(dtype=0, rows=3, cols=8, x=P, ldx=8, weight=P, mean=P, rstd=P, dy=P, lddy=8, dx=P,
              lddx=8, dweight=P, dbias=P, ws=P, ws_bytes=1 << 20, stream=None)
LINEAR = dict(dtype=0, rows=3, n_in=8, n_out=5, x=P, ldx=8, weight=P, ldw=8, bias=P, act=1,
              residual=P, ldr=5, y=P, ldy=5, pre=P, ws=P, ws_bytes=1 << 20, stream=None)
LINEAR_B = dict(dtype=0, rows=3, n_in=8, n_out=5, x=P, ldx=8, weight=P, ldw=8, act=1, pre=P, dy=P,
                lddy=5, dx=P, lddx=8, dweight=P, lddw=8, dbias=P, ws=P, ws_bytes=1 << 20,
                stream=None)
SCORES = dict(kind=0, dtype=0, rows=3, cols=8, scores=P, lds=8, inv_t=1.0, targets=P, n_targets=1,
              logp=P, entropy=P, n_top=2, top_logp=P, top_index=P, stats=P, ws=P, ws_bytes=1 << 20,
              stream=None)
SCORES_B = dict(dtype=0, rows=3, cols=8, scores=P, lds=8, inv_t=1.0, targets=P, n_targets=1,
                stats=P, entropy=P, dlogp=P, dentropy=P, dscores=P, ldds=8, stream=None)
INV, BIG, WS = _lib.VQC_ERR_INVALID_ARG, _lib.VQC_ERR_TOO_LARGE, _lib.VQC_ERR_WORKSPACE

REFUSED = [
    ("vqc_layer_norm", NORM, [
        (dict(dtype=3), INV), (dict(rows=-1), INV), (dict(cols=0), INV), (dict(eps=-1.0), INV),
        (dict(eps=NAN), INV), (dict(eps=INF), INV), (dict(x=None), INV), (dict(y=None), INV),
        (dict(x=P + 2), INV), (dict(y=P + 1), INV), (dict(weight=P + 2), INV), (dict(ldy=7), INV),
        (dict(ldx=-8), INV), (dict(mean=None), INV), (dict(rstd=None), INV),
        (dict(dtype=2, x=P + 1), INV), (dict(rows=1 << 41), BIG),
        (dict(rows=1 << 30, cols=1 << 20), BIG), (dict(ldx=1 << 62), BIG)]),
    ("vqc_layer_norm_backward", NORM_B, [
        (dict(dtype=-1), INV), (dict(cols=0), INV), (dict(dy=None), INV), (dict(mean=None), INV),
        (dict(rstd=None), INV), (dict(lddx=4), INV), (dict(ws=None), WS), (dict(ws=P + 8), WS),
        (dict(ws_bytes=16), WS), (dict(dweight=P + 2), INV)]),
    ("vqc_linear", LINEAR, [
        (dict(dtype=9), INV), (dict(act=5), INV), (dict(act=-1), INV), (dict(n_in=-1), INV),
        (dict(x=None), INV), (dict(weight=None), INV), (dict(y=None), INV), (dict(ldy=4), INV),
        (dict(ldw=-1), INV), (dict(pre=P + 2), INV), (dict(residual=P + 1), INV),
        (dict(rows=1 << 39, n_out=4), BIG)]),
    ("vqc_linear_backward", LINEAR_B, [
        (dict(pre=None), INV), (dict(dy=None), INV), (dict(x=None), INV), (dict(weight=None), INV),
        (dict(lddx=7), INV), (dict(lddw=7), INV), (dict(ws=None), WS), (dict(ws_bytes=0), WS),
        (dict(ws=P + 128), WS)]),
    ("vqc_log_probs", SCORES, [
        (dict(kind=2), INV), (dict(dtype=5), INV), (dict(cols=0), INV), (dict(inv_t=0.0), INV),
        (dict(inv_t=NAN), INV), (dict(inv_t=INF), INV), (dict(kind=1, inv_t=2.0), INV),
        (dict(n_top=9), INV), (dict(cols=100, n_top=65), INV), (dict(n_top=-1), INV),
        (dict(scores=None), INV), (dict(targets=None), INV), (dict(logp=None), INV),
        (dict(top_logp=None), INV), (dict(top_index=None), INV), (dict(top_index=P + 4), INV),
        (dict(rows=1, cols=1 << 31), BIG), (dict(n_targets=-1), INV),
        (dict(rows=1, cols=1 << 20, lds=1 << 20, ws=None), WS)]),
    ("vqc_log_probs_backward", SCORES_B, [
        (dict(stats=None), INV), (dict(entropy=None), INV), (dict(dscores=None), INV),
        (dict(ldds=7), INV), (dict(targets=None), INV), (dict(inv_t=-1.0), INV),
        (dict(scores=P + 2), INV)]),
]


@pytest.mark.parametrize("name,good,change,status",
                         [(n, g, c, s) for n, g, cs in REFUSED for c, s in cs],
                         ids=lambda v: str(v) if isinstance(v, (str, int)) else "-".join(
                             f"{k}={x}" for k, x in v.items()) if len(v) < 5 else "")
def test_refused(lib, name, good, change, status):
    assert getattr(lib, name)(*{**good, **change}.values()) == status
    assert _lib.vqc_last_error()


def test_empty_calls_launch_nothing(lib):
    assert lib.vqc_layer_norm(*{**NORM, "rows": 0, "x": None, "y": None}.values()) == 0
    assert lib.vqc_layer_norm_backward(*{**NORM_B, "dx": None, "dweight": None,
                                         "dbias": None}.values()) == 0
    assert lib.vqc_linear(*{**LINEAR, "rows": 0, "x": None, "y": None}.values()) == 0
    assert lib.vqc_linear(*{**LINEAR, "n_out": 0, "weight": None, "y": None}.values()) == 0
    assert lib.vqc_linear_backward(*{**LINEAR_B, "dx": None, "dweight": None,
                                     "dbias": None}.values()) == 0
    assert lib.vqc_log_probs(*{**SCORES, "rows": 0, "scores": None}.values()) == 0
    assert lib.vqc_log_probs_backward(*{**SCORES_B, "rows": 0, "scores": None}.values()) == 0


def test_workspace_sizes(lib):
    bad = ctypes.c_size_t(-1).value
    assert lib.vqc_layer_norm_workspace_bytes(-1, 4) == bad
    assert lib.vqc_layer_norm_workspace_bytes(3, 0) == bad
    assert lib.vqc_layer_norm_workspace_bytes(0, 4) == 0
    assert lib.vqc_layer_norm_workspace_bytes(100, 40) > 0
    assert lib.vqc_linear_workspace_bytes(3, 1, 1, 1, 0) == bad
    assert lib.vqc_linear_workspace_bytes(0, 1, 1, 1, 2) == bad
    assert lib.vqc_linear_workspace_bytes(0, -1, 1, 1, 0) == bad
    assert lib.vqc_linear_workspace_bytes(0, 0, 0, 0, 0) == 0
    assert lib.vqc_log_probs_workspace_bytes(1, 4, 5) == bad
    assert lib.vqc_log_probs_workspace_bytes(1000, 100, 5) == 0
    assert lib.vqc_log_probs_workspace_bytes(1, 1 << 20, 5) > 0
    # sizes that would overflow are refused, not wrapped
    assert lib.vqc_layer_norm_workspace_bytes(1 << 40, 1 << 40) == bad
    assert lib.vqc_linear_workspace_bytes(0, 1 << 40, 1 << 40, 1 << 40, 1) == bad
