"""Rows and linear layers in 8-bit integers on the GPU against plain 64-bit forms
(serving_oracle.py)."""
import math

import pytest
import torch

from tests import layers_oracle as O
from tests import serving_oracle as S
from tests.test_gpu_layers import ACTS, DEV, TYPES, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_amd import layers as m
    return m


# ------------------------------------------------------------------ quantize

ROWS = [(1, 1), (3, 2), (5, 3), (7, 8), (64, 16), (7, 255), (33, 257), (16, 1000), (9, 1025),
        (4, 4096), (9, 4097), (2, 16384), (3, 16385), (2, 40001), (300, 40),
        (257, 4097), (300, 8192), (258, 8193), (300, 16383), (261, 16384)]


def same_integers(got, x):
    q, s = S.quantized(x)
    assert got.values.shape == q.shape and got.scales.shape == s.shape
    assert got.values.dtype == torch.int8 and got.scales.dtype == torch.float32
    assert torch.equal(got.values.cpu(), q)
    torch.testing.assert_close(got.scales.cpu(), s, rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", ROWS)
def test_quantize(layers, rows, cols, dtype):
    x = rand((rows, cols), rows + cols, dtype, 1.5, pad=cols % 4)
    same_integers(layers.quantize(x), x)


@pytest.mark.parametrize("dtype,scale", [(torch.float32, 0), (torch.float32, 119),
                                         (torch.float32, -130), (torch.float16, 0),
                                         (torch.bfloat16, 0), (torch.bfloat16, 119),
                                         (torch.bfloat16, -118)], ids=str)
def test_quantize_ties_and_borders(layers, dtype, scale):
    """Exact ties go to the even integer, numbers one place beside them to the nearest, in rows of
    ordinary, of the largest and of small numbers."""
    eps = torch.finfo(dtype).eps
    x = torch.zeros((6, 600))
    x[0, 0], x[1, 0] = 1.0, 254.0
    x[2, 0], x[3, 0] = -127.0, 96.0
    x[4, 0], x[5, 0] = 1.9921875, 3.0
    halves = (torch.arange(1, 254, 2).float() / 254).repeat(2)[:250]
    for r in range(6):
        base = halves * x[r, 0].abs()
        x[r, 1:251] = base
        x[r, 251:501] = -base * (1 + eps)
    x[0, 501:520] = 0.5
    x = (x * 2.0 ** (scale // 2) * 2.0 ** (scale - scale // 2)).to(dtype).to(DEV)
    assert torch.isfinite(x).all()
    same_integers(layers.quantize(x), x)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols", [5, 300, 20000])
def test_quantize_rows_of_every_size(layers, cols, dtype):
    """Zeros, the smallest and the largest numbers, infinities and NaN, each in its own row."""
    x = rand((9, cols), 3, torch.float32)
    f = torch.finfo(dtype)
    x[1] = 0
    x[2] *= f.smallest_normal * 2.0 ** -4
    x[3] *= f.smallest_normal * 0.4
    x[4] *= f.max / 8
    x[7] = 0
    x[7, 2] = f.smallest_normal * f.eps
    x = x.to(dtype)
    x[5, cols // 2] = math.nan
    x[6, cols - 1] = -math.inf
    got = layers.quantize(x)
    same_integers(got, x)
    assert got.scales[5:7].isnan().all() and not got.scales[[0, 1, 2, 3, 4, 7, 8]].isnan().any()


def test_quantize_shapes(layers):
    x = rand((2, 3, 5, 37), 4, torch.bfloat16)
    got = layers.quantize(x)
    assert got.values.shape == x.shape and got.scales.shape == x.shape[:-1]
    same_integers(got, x)
    one = layers.quantize(rand((40,), 5, torch.float32))
    assert one.values.shape == (40,) and one.scales.shape == ()
    for shape in ((0, 5), (3, 0), (0, 0), (2, 0, 4)):
        got = layers.quantize(torch.empty(shape, device=DEV))
        assert got.values.shape == shape and got.scales.shape == shape[:-1]
        assert (got.scales == 0).all()
    # one row for all, and rows in falling order of their addresses' distance
    base = rand((1, 50), 6, torch.float16)
    same_integers(layers.quantize(base.expand(7, 50)), base.expand(7, 50))


def test_quantize_writes_nothing_behind_a_row(layers):
    """Through the C entry: integers of rows 16 apart from each other stay within theirs."""
    from paper_2607_11985_amd import _lib
    x = rand((5, 21), 7, torch.float16)
    q = torch.full((5, 40), 99, dtype=torch.int8, device=DEV)
    s = torch.full((6,), -1.0, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    _lib._check(_lib.load().vqc_quantize(1, 5, 21, x.data_ptr(), 21, q.data_ptr() + 1, 40,
                                         s.data_ptr(), stream))
    want, steps = S.quantized(x)
    assert torch.equal(q[:, 1:22].cpu(), want) and torch.equal(s[:5].cpu(), steps)
    assert (q[:, 0] == 99).all() and (q[:, 22:] == 99).all() and s[5] == -1


# ------------------------------------------------------------------ linear

SIZES = [(1, 1, 1), (1, 16, 10), (64, 16, 10), (3, 5, 7), (1, 300, 77), (2, 4096, 130),
         (5, 1000, 64), (8, 513, 9), (4, 1024, 4100), (17, 129, 65), (65, 64, 63), (33, 2048, 16),
         (130, 40, 257), (256, 256, 256), (300, 520, 300), (1, 5000, 1), (700, 3, 2),
         (16, 64, 4100), (513, 1040, 264), (9, 4096, 512), (40, 8192, 96), (300, 16384, 101),
         # one row: more columns than workgroups, the two longer forms
         (1, 2500, 9000), (1, 6000, 70), (1, 16384, 33), (1, 16385, 9),
         # up to eight pieces of 1024, every length
         (1, 300, 9000), (8, 1000, 50), (4, 2048, 40), (2, 4000, 30), (8, 256, 16), (7, 777, 90),
         # few rows: more columns than workgroups, 32 rows, every length
         (3, 512, 9000), (25, 400, 40), (20, 2000, 33), (32, 3000, 50), (32, 4096, 17),
         (31, 4097, 20), (33, 700, 20),
         # short rows: every length, more columns than a workgroup's waves
         (8000, 16, 600), (50, 200, 300), (90, 300, 130), (40, 600, 70), (40, 1000, 90),
         (40, 1024, 33), (40, 1025, 33),
         # the largest tiles, whole and at the edges
         (1990, 600, 7003), (600, 9000, 600),
         # the tiles between, at the edges
         (2040, 1030, 1910)]


def case(rows, n_in, n_out, dtype, seed):
    x = rand((rows, n_in), seed, dtype, 1.3, pad=(rows + n_in) % 3)
    w = rand((n_out, n_in), seed + 1, torch.float32, n_in ** -0.5)
    b = rand((n_out,), seed + 2, dtype, 0.3)
    r = rand((rows, n_out), seed + 3, dtype, pad=n_out % 2)
    return x, w, b, r


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
def test_linear(layers, rows, n_in, n_out, dtype):
    x, w, b, r = case(rows, n_in, n_out, dtype, 10)
    name = ACTS[(rows + n_in + n_out) % len(ACTS)]
    w8 = layers.quantize(w)
    y = layers.linear_quantized(x, w8, b, name, r)
    assert y.dtype == dtype and y.shape == (rows, n_out)
    xq, xs = S.quantized(x)
    want, bound = S.linear(xq, xs, w8.values, w8.scales, O.d(b), name, O.d(r))
    O.check(y, want, bound, dtype, name)
    # the rows as integers beforehand: the same numbers
    y8 = layers.linear_quantized(layers.quantize(x), w8, b, name, r, dtype=dtype)
    assert torch.equal(y8, y)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_linear_activations(layers, dtype, name):
    for rows, n_in, n_out in ((3, 700, 50), (70, 130, 90)):
        x, w, b, r = case(rows, n_in, n_out, dtype, 20)
        w8 = layers.quantize(w)
        xq, xs = S.quantized(x)
        for bias, residual in ((None, None), (b, None), (None, r)):
            y = layers.linear_quantized(x, w8, bias, name, residual)
            want, bound = S.linear(xq, xs, w8.values, w8.scales, O.d(bias), name, O.d(residual))
            O.check(y, want, bound, dtype, name)


# (rows, n_in, n_out) of every kernel: row by row, tiles of 32, 64, 128 and 256, splits of k
EXACT = [(1, 4096, 40), (7, 1500, 33), (8, 600, 70), (20, 100, 30), (30, 3000, 70), (64, 4096, 128),
         (200, 300, 200), (1000, 512, 1024), (2048, 1024, 2048), (2304, 500, 2560),
         (1990, 1000, 7001), (600, 9000, 600), (128, 20000, 256), (3, 140000, 5), (70, 300000, 40),
         # splits of every tile
         (66, 3330, 8241), (131, 11040, 6333)]


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("rows,n_in,n_out", EXACT)
def test_sums_are_exact(layers, rows, n_in, n_out, aligned):
    """Whole numbers, -128 among them, in rows on and off the 16-byte chunks: the result is the sum
    rounded to fp32 once, bit for bit, however it is put together."""
    g = torch.Generator().manual_seed(rows + n_out)

    def ints(n):
        ld = (n_in + 15) // 16 * 16 + (0 if aligned else 3)
        t = torch.randint(-128, 128, (n, ld), generator=g, dtype=torch.int8)
        t[:, n_in:] = 111  # what lies behind a row takes no part
        t[0, :n_in] = -128
        return t.to(DEV)[:, :n_in]

    xq, wq = ints(rows), ints(n_out)
    one = lambda n: torch.ones(n, device=DEV)
    y = layers.linear_quantized(layers.Quantized(xq, one(rows)), layers.Quantized(wq, one(n_out)))
    sums = S.products(xq, wq)
    assert torch.equal(y.cpu(), sums.float())
    assert float(sums.max()) >= 128 * 128 * n_in
    # the row's step, then the channel's
    xs, ws = torch.rand(rows, generator=g) * 1e-3, torch.rand(n_out, generator=g) + 0.1
    y = layers.linear_quantized(layers.Quantized(xq, xs.to(DEV)), layers.Quantized(wq, ws.to(DEV)))
    assert torch.equal(y.cpu(), sums.float() * xs[:, None] * ws)


def test_linear_rows_are_apart(layers):
    """NaN and infinities stay in their rows and channels."""
    for rows in (4, 40):
        x, w, b, _ = case(rows, 600, 30, torch.float32, 30)
        y0 = layers.linear_quantized(x, layers.quantize(w), b)
        z, v = x.clone(), w.clone()
        z[1, 5], v[7, 0] = math.inf, math.nan
        y1 = layers.linear_quantized(z, layers.quantize(v), b)
        keep = torch.ones((rows, 30), dtype=torch.bool, device=DEV)
        keep[1], keep[:, 7] = False, False
        assert torch.equal(y1[keep], y0[keep]) and y1[~keep].isnan().all()


def test_linear_empty(layers):
    w8 = layers.quantize(rand((4, 6), 1, torch.float32))
    b = rand((4,), 2, torch.float32)
    assert layers.linear_quantized(torch.empty((0, 6), device=DEV), w8, b).shape == (0, 4)
    none = layers.quantize(torch.empty((0, 6), device=DEV))
    assert layers.linear_quantized(rand((3, 6), 3, torch.float32), none).shape == (3, 0)
    flat = layers.quantize(torch.empty((4, 0), device=DEV))
    y = layers.linear_quantized(torch.empty((3, 0), device=DEV), flat, b)
    assert torch.equal(y, b.expand(3, 4))


def test_linear_shapes_and_strides(layers):
    x = rand((2, 5, 3, 48), 40, torch.bfloat16)
    w8 = layers.quantize(rand((20, 48), 41, torch.float32))
    r = rand((2, 5, 3, 20), 42, torch.bfloat16)
    y = layers.linear_quantized(x, w8, None, "none", r)
    flat = layers.linear_quantized(x.reshape(30, 48), w8, None, "none", r.reshape(30, 20))
    assert y.shape == (2, 5, 3, 20) and torch.equal(y.reshape(30, 20), flat)
    # integers of a batch, a single row, one row for all, every second row
    assert torch.equal(layers.linear_quantized(layers.quantize(x), w8, None, "none", r,
                                               dtype=torch.bfloat16), y)
    one = layers.linear_quantized(x[0, 0, 0], w8)
    assert one.shape == (20,)
    assert torch.equal(layers.linear_quantized(x[0, 0, :1].expand(9, 48), w8),
                       one.expand(9, 20))
    assert torch.equal(layers.linear_quantized(x.reshape(30, 48)[::2], w8),
                       layers.linear_quantized(x.reshape(30, 48), w8)[::2])
    # scales out of a wider table
    wide = torch.stack([w8.scales, w8.scales], 1)[:, 0]
    assert torch.equal(layers.linear_quantized(x, layers.Quantized(w8.values, wide)),
                       layers.linear_quantized(x, w8))


def test_linear_near_the_layer_it_stands_for(layers):
    """Against the layer in 32 bits: every product is off by half a step of each side at most."""
    x, w, b, r = case(60, 500, 70, torch.float32, 50)
    w8 = layers.quantize(w)
    y = layers.linear_quantized(x, w8, b, "none", r)
    want = layers.linear(x, w, b, "none", r)
    xd, wd = O.d(x), O.d(w)
    sx, sw = xd.abs().amax(1, keepdim=True) / 254, wd.abs().amax(1) / 254
    limit = sx * wd.abs().sum(1) + sw * xd.abs().sum(1, keepdim=True) + 500 * sx * sw
    assert (O.d(y - want).abs() <= limit + 1e-4).all()


def test_refusals(layers):
    x, w, b, r = case(4, 32, 6, torch.float32, 60)
    w8 = layers.quantize(w)
    lin = layers.linear_quantized
    bad = [
        lambda: layers.quantize(x.cpu()), lambda: layers.quantize(x.double()),
        lambda: layers.quantize(x.T), lambda: layers.quantize(torch.tensor(1.0, device=DEV)),
        lambda: layers.quantize(x.detach().clone().requires_grad_(True)),
        lambda: lin(x, w8, b, "sigmoid"), lambda: lin(x[:, :31], w8),
        lambda: lin(x, layers.Quantized(w, w8.scales)),
        lambda: lin(x, layers.Quantized(w8.values, w8.scales[:5])),
        lambda: lin(x, layers.Quantized(w8.values, w8.scales.double())),
        lambda: lin(x, layers.Quantized(w8.values.cpu(), w8.scales)),
        lambda: lin(x, layers.Quantized(w8.values[0], w8.scales[0])),
        lambda: lin(x, w8, b.half()), lambda: lin(x, w8, b[:5]),
        lambda: lin(x, w8, b, "none", r[:3]), lambda: lin(x, w8, b, "none", r.half()),
        lambda: lin(x.half(), w8, None, "none", None, torch.float32),
        lambda: lin(layers.quantize(x), w8, dtype=torch.float64),
        lambda: lin(layers.quantize(x), w8, b.half()),
        lambda: lin(layers.Quantized(w8.values, torch.ones(4, device=DEV)), w8),
        lambda: lin(x.detach().clone().requires_grad_(True), w8),
        lambda: lin(x, w8, b.detach().clone().requires_grad_(True)),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was let through")
    with torch.no_grad():
        v = x.detach().clone().requires_grad_(True)
        assert torch.equal(lin(v, w8, b), lin(x, w8, b))


def test_streams_and_graphs(layers):
    """On another stream, and captured: two graphs replayed in turn with eager calls between."""
    x, w, b, r = case(5, 2048, 96, torch.bfloat16, 70)
    big, _, _, _ = case(200, 2048, 96, torch.bfloat16, 71)
    w8 = layers.quantize(w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = layers.linear_quantized(x, w8, b, "gelu", r)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, layers.linear_quantized(x, w8, b, "gelu", r))
    graphs = []
    for v in (x, big):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layers.linear_quantized(v, w8, b, "silu")
        graphs.append((g, v, out))
    for k in range(3):
        for g, v, out in graphs:
            v.copy_(rand(v.shape, 80 + k, torch.bfloat16))
            g.replay()
            want = layers.linear_quantized(v, w8, b, "silu")
            torch.cuda.synchronize()
            assert torch.equal(out, want)


# ------------------------------------------------------------------ offsets beyond 32 bits

def test_long_operands(layers):
    """More than 2^32 bytes of x, W or y: the ends of the whole are those of a part."""
    g = torch.Generator(device=DEV).manual_seed(8)

    def integers(rows, cols):
        return layers.Quantized(
            torch.randint(-128, 128, (rows, cols), generator=g, device=DEV, dtype=torch.int8),
            torch.rand(rows, generator=g, device=DEV) + 0.5)

    def last(q, n):
        return layers.Quantized(q.values[-n:].clone(), q.scales[-n:].clone())
    long, short = integers(70000, 65536), integers(33, 65536)
    for wide in (False, True):  # rows on 16 bytes and off them
        a, b = long, short
        if wide:
            a, b = (layers.Quantized(q.values[:, 1:], q.scales) for q in (long, short))
        y = layers.linear_quantized(b, a)
        assert torch.equal(y[:, -100:], layers.linear_quantized(b, last(a, 100)))
        y = layers.linear_quantized(a, b)
        assert torch.equal(y[-100:], layers.linear_quantized(last(a, 100), b))
    few = layers.Quantized(short.values[:3, :4096], short.scales[:3])  # rows 65536 apart
    part = layers.Quantized(long.values[:, -4096:], long.scales)
    y = layers.linear_quantized(few, part)
    assert torch.equal(y[:, -100:], layers.linear_quantized(few, last(part, 100)))
    del long, short, part
    x = torch.randn((40000, 65536), generator=g, device=DEV, dtype=torch.bfloat16)
    got, want = layers.quantize(x), layers.quantize(x[-50:].clone())
    assert torch.equal(got.values[-50:], want.values) and torch.equal(got.scales[-50:], want.scales)
    del x, got
    x = torch.randn((70000, 64), generator=g, device=DEV, dtype=torch.float16)
    w = layers.quantize(torch.randn((70000, 64), generator=g, device=DEV))
    y = layers.linear_quantized(x, w, residual=None)
    assert torch.equal(y[-70:, -90:], layers.linear_quantized(x[-70:], last(w, 90)))
    y = layers.linear_quantized(x, w, residual=y)
    assert torch.equal(y[-70:, -90:], layers.linear_quantized(
        x[-70:], last(w, 90), residual=layers.linear_quantized(x[-70:], last(w, 90))))
