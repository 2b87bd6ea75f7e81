"""Linear layers through the larger tiles' main loops and the copies onto 16-byte chunks, against
products in 64 bits on the GPU (sizes in layers_tiles.py, bounds in layers_oracle.py)."""
import math

import pytest
import torch

from tests import layers_oracle as O
from tests import layers_tiles as T
from tests.test_gpu_layers import DEV, TYPES, grads_of, linear_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_amd import layers as m
    return m


def near(got, want, bound, dtype, what):
    err = (got.detach().double() - want).abs()
    limit = O.ROUND[dtype] * want.abs() + O.TINY[dtype] + bound
    bad = ~(err <= limit)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound"


def check(layers, x, w, b, r, dy, name):
    """All outputs of a forward and backward; the calls' results twice the same."""
    dtype = x.dtype
    ins = [v.detach().requires_grad_(True) for v in (x, w, b)]
    y = layers.linear(*ins, name, r)
    grads = grads_of(y, ins, dy)
    xd, wd, bd, rd, dyd = (v.detach().double() for v in (x, w, b, r, dy))
    near(y, O.linear(xd, wd, bd, name, rd)[0], O.linear_bounds(xd, wd, bd, name, rd)[0], dtype, "y")
    for got, want, bound, what in zip(grads, O.linear_grads(xd, wd, bd, name, dyd),
                                      O.linear_grad_bounds(xd, wd, bd, name, dyd, dtype),
                                      ("dx", "dw", "db")):
        near(got, want, bound, dtype, what)
    y2 = layers.linear(*ins, name, r)
    assert torch.equal(y2, y)
    for a, c in zip(grads_of(y2, ins, dy), grads):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("which", [0, 1, 2], ids=["forward", "dx", "dweight"])
@pytest.mark.parametrize("k", range(4))
def test_larger_tiles(layers, k, which, dtype):
    size = [s for e, s, _, _ in T.PRODUCTS if e == dtype.itemsize][k]
    case = (v.contiguous() for v in linear_case(*T.layer_of(which, *size), dtype, "silu", 110))
    check(layers, *case, "tanh")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("name", ["none", "gelu"])
@pytest.mark.parametrize("size", [s for s, _ in T.COPIED], ids=str)
def test_copied_rows(layers, size, name, dtype):
    """Odd widths: every row starts at another offset from the chunks."""
    check(layers, *(v.contiguous() for v in linear_case(*size, dtype, name, 111)), name)


def framed(v, before, stride):
    """The same rows in a table of NaN, `before` elements in and `stride` apart."""
    rows, cols = v.shape
    t = torch.full((rows + 2, stride), math.nan, dtype=v.dtype, device=DEV)
    t[1:-1, before:before + cols] = v
    return t[1:-1, before:before + cols]


# elements before a row and behind it: views of one odd offset and an odd stride, of a stride on the
# chunks, and of a start on them
FRAMES = [(1, 2), (3, 8), (0, 7), (0, 1), (5, 0), (8, 8)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("before,behind", FRAMES)
@pytest.mark.parametrize("name", ["none", "tanh"])
@pytest.mark.parametrize("size", [(1409, 1201, 1303), (1408, 1200, 1304)], ids=str)
def test_strided_rows(layers, size, name, before, behind, dtype):
    """Tables whose rows lie between NaN, at offsets and strides on and off the chunks, with widths
    that divide them and others: none of the NaN in any result."""
    x, w, b, r, dy = (v.contiguous() for v in linear_case(*size, dtype, name, 112))
    x, w, r, dy = (framed(v, before, before + v.shape[1] + behind) for v in (x, w, r, dy))
    check(layers, x, w, b, r, dy, name)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_stride_on_the_chunks_and_odd_width(layers, dtype):
    """Rows on the chunks whose last chunk is not full, read by columns."""
    x, w, b, r, dy = (v.contiguous() for v in linear_case(1409, 1201, 1303, dtype, "none", 113))
    x, w, r, dy = (framed(v, 8, (v.shape[1] + 15) // 8 * 8) for v in (x, w, r, dy))
    for name in ("none", "silu"):
        check(layers, x, w, b, r, dy, name)
