"""Layers at the ends of their ranges."""

import pytest
import torch

from tests import layers_oracle as O
from tests.test_gpu_layers import DEV, grads_of, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_amd import layers as m
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("cols", [1, 3, 5, 77, 250, 259, 1000, 4095, 5001, 16383, 16385])
def test_layer_norm_gradient_of_large_constant_rows(layers, cols, dtype):
    """Rows of 2^112, whose mean is exact: h = 0, though mean * rstd is beyond fp32, and what lies
    behind a row's end takes no part.  dx = rstd (g - mean g), dw = 0."""
    eps = 1e-16
    x = torch.full((3, cols), 2.0 ** 112, dtype=dtype, device=DEV).requires_grad_(True)
    w, b = (rand((cols,), s, dtype).requires_grad_(True) for s in (1, 2))
    dy = rand((3, cols), 3, dtype)
    y = layers.layer_norm(x, w, b, eps)
    dx, dw, db = grads_of(y, (x, w, b), dy)
    assert torch.equal(y, b.expand(3, cols)) and (dw == 0).all()
    g = O.d(dy) * O.d(w)
    rstd = float(torch.tensor(eps, dtype=torch.float32).double()) ** -0.5
    mean = g.mean(-1, keepdim=True)
    # a sum of g in fp32 (log-depth), rstd's own few roundings
    bound = 64 * O.U * rstd * (g.abs() + g.abs().mean(-1, keepdim=True))
    O.check(dx, rstd * (g - mean), bound, dtype, "dx")
    O.check(db, O.d(dy).sum(0), 16 * O.U * O.d(dy).abs().sum(0), dtype, "db")
