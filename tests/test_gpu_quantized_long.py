"""Linear layers in 8-bit integers with more rows than one grid holds."""
import pytest
import torch

from tests import serving_oracle as S
from tests import layers_oracle as O
from tests.test_gpu_layers import DEV, TYPES
from tests.test_gpu_quantized import layers  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

GRID = (2 ** 31 - 1) // 512 * 16  # rows of a launch of the kernel for short ones


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_more_short_rows_than_a_grid_holds(layers, dtype):
    """On both sides of where a launch ends and at the ends, against the plain form; the rest against
    calls of its parts."""
    n_in = 16 // dtype.itemsize
    rows = 75_000_000 if n_in == 4 else GRID + 37
    g = torch.Generator(device=DEV).manual_seed(n_in)
    x = torch.randn((rows, n_in), generator=g, device=DEV).to(dtype)
    r = torch.randn((rows, 1), generator=g, device=DEV).to(dtype)
    w8 = layers.quantize(torch.randn((1, n_in), generator=g, device=DEV))
    b = torch.randn((1,), generator=g, device=DEV).to(dtype)
    y = layers.linear_quantized(x, w8, b, "silu", r)
    assert y.shape == (rows, 1)
    for a in (0, GRID - 40, rows - 40):
        part = slice(a, a + 40)
        xq, xs = S.quantized(x[part])
        want, bound = S.linear(xq, xs, w8.values, w8.scales, O.d(b), "silu", O.d(r[part]))
        O.check(y[part], want, bound, dtype, "silu")
    half = rows // 2
    for part in (slice(0, half), slice(half, rows)):
        assert torch.equal(y[part], layers.linear_quantized(x[part], w8, b, "silu", r[part]))


def test_more_integers_than_a_grid_pads(layers):
    """Rows given as integers that do not end with a stage of k are copied to ones that do: 2^28 + 5000 of
    them, 2^35 bytes, are more than one launch takes."""
    rows = 2 ** 28 + 5000
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-128, 128, (rows, 1), generator=g, device=DEV, dtype=torch.int8)
    s = torch.rand((rows,), generator=g, device=DEV)
    w = layers.Quantized(torch.tensor([[-128]], dtype=torch.int8, device=DEV),
                         torch.tensor([0.37], device=DEV))
    y = layers.linear_quantized(layers.Quantized(x, s), w, dtype=torch.float16)
    for a in range(0, rows, 2 ** 26):  # an exact product, and two of fp32 one after the other
        part = slice(a, min(rows, a + 2 ** 26))
        want = (x[part].float() * -128 * s[part, None] * 0.37).half()
        assert torch.equal(y[part], want)
