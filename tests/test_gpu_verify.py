"""Verification of drafted outcomes on the GPU against plain 64-bit sums (serving_oracle.py)."""
import math

import pytest
import torch

from tests import serving_oracle as S
from tests.test_gpu_layers import DEV, TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_amd import layers as m
    return m


def case(n, k, cols, dtype, seed, kind="logits", near=0.7):
    """Target and draft alike, drafts drawn from the draft, and uniform numbers."""
    g = torch.Generator().manual_seed(seed)
    t = 2 * torch.randn((n, k + 1, cols), generator=g)
    q = t[:, :k] + near * torch.randn((n, k, cols), generator=g)
    if kind == "weights":
        t, q = torch.softmax(t, -1) * 3, torch.softmax(q, -1)
    t, q = t.to(dtype), q.to(dtype)
    p = q.double() if kind == "weights" else torch.softmax(q.double(), -1)
    if k:
        d = torch.multinomial(p.reshape(n * k, cols), 1, generator=g).reshape(n, k)
    else:
        d = torch.empty((n, 0), dtype=torch.int64)
    u = torch.rand((n, k + 1), generator=g, dtype=torch.float64)
    return t.to(DEV), q.to(DEV), d.to(DEV), u.to(DEV)


def same(got, want):
    assert got.outcomes.dtype == torch.int64 and got.accepted.dtype == torch.int64
    assert torch.equal(got.accepted.cpu(), want[1]), (got.accepted, want[1])
    assert torch.equal(got.outcomes.cpu(), want[0])


SIZES = [(1, 0, 1), (3, 1, 1), (1, 1, 2), (5, 2, 3), (4, 3, 7), (1, 3, 1024), (16, 4, 255),
         (9, 5, 257), (3, 1, 2048), (2, 2, 2049), (6, 0, 5000), (4, 7, 5001), (1, 2, 40000),
         (2, 1, 131077), (300, 2, 50), (2, 19, 64),
         # more rows than one workgroup keeps, one unit of the drawn row
         (3, 40, 300), (2, 70, 5),
         # rows behind a refused draft are passed over; several packs for each lane
         # (passed over at the last of them, the first two have too few scores and no drafts)
         (64, 4, 33000), (300, 0, 40000), (110, 6, 50000)]


@pytest.mark.parametrize("kind", ["logits", "weights"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,k,cols", SIZES)
def test_verify(layers, n, k, cols, dtype, kind):
    t, q, d, u = case(n, k, cols, dtype, n + k + cols, kind)
    temperature = 1.0 if kind == "weights" else (1.0, 0.5, 1.3)[cols % 3]
    got = layers.verify_drafts(t, q, d, u, kind, temperature)
    same(got, S.verify(t, q, d, u, kind, temperature))
    # drafts that were certain
    same(layers.verify_drafts(t, None, d, u, kind, temperature),
         S.verify(t, None, d, u, kind, temperature))


@pytest.mark.parametrize("cols", [5, 3000, 60001])
def test_every_place_is_reached(layers, cols):
    """The drafts stand or fall where the uniform numbers say, and the outcome behind them is the
    first and the last with any weight at the ends of [0, 1)."""
    n, k = 12, 4
    t, q, d, u = case(n, k, cols, torch.float32, cols)
    u[:, :k] = 0
    for s in range(n):
        if s % (k + 2) <= k:
            u[s, s % (k + 2):k] = 1 - 2.0 ** -53
    q[:, :, :] = t[:, :k]
    q.scatter_add_(2, d[..., None], torch.ones((n, k, 1), device=DEV))
    u[:, k] = torch.tensor([0, 1 - 2.0 ** -53, 0.5] * 4, device=DEV, dtype=torch.float64)
    want = S.verify(t, q, d, u)
    assert set(want[1].tolist()) == set(range(k + 1))
    same(layers.verify_drafts(t, q, d, u), want)


def test_equal_weights_and_borders(layers):
    """Sums that are exact: a uniform number on a border belongs to the outcome behind it."""
    for cols in (8, 4096, 65536):
        n = 64
        t = torch.full((n, 1, cols), 0.25, device=DEV)
        u = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] / n
        d = torch.empty((n, 0), dtype=torch.int64, device=DEV)
        for kind in ("weights", "logits"):
            got = layers.verify_drafts(t, None, d, u, kind)
            assert torch.equal(got.outcomes[:, 0], torch.arange(n, device=DEV) * cols // n)
            assert (got.accepted == 0).all()


def test_drafts_that_end_early(layers):
    """-1 and any other index outside the row ends the drafts; what is behind is not looked at."""
    t, q, d, u = case(8, 4, 500, torch.float16, 5)
    q.copy_(t[:, :4])  # the same: every draft is accepted
    for s, bad in enumerate((-1, 500, -(2 ** 63), 2 ** 63 - 1)):
        d[s, s] = bad
    q[0, 1:], t[1, 2:] = math.nan, math.nan
    got = layers.verify_drafts(t, q, d, u)
    same(got, S.verify(t, q, d, u))
    assert got.accepted.tolist() == [0, 1, 2, 3, 4, 4, 4, 4]
    assert (got.outcomes[0, 0] >= 0) and (got.outcomes[0, 1:] == -1).all()


@pytest.mark.parametrize("n,k,cols", [(3, 2, 7), (4, 3, 4000), (4, 3, 70000), (64, 4, 33000)])
@pytest.mark.parametrize("mask", [-math.inf, torch.finfo(torch.float32).min])
def test_drafts_without_a_share(layers, mask, n, k, cols):
    """A uniform number of 0 accepts whatever has a share, and nothing that has none."""
    t, q, d, u = case(n, k, cols, torch.float32, n + k + cols)
    u[:, :k] = 0
    ends = torch.arange(n, device=DEV) % (k + 1)
    for s in range(n):
        if ends[s] < k:
            t[s, ends[s], d[s, ends[s]]] = mask
            if s % 2:  # nor of the draft's
                q[s, ends[s], d[s, ends[s]]] = mask
    for draft in (q, None):
        got = layers.verify_drafts(t, draft, d, u)
        assert torch.equal(got.accepted, ends)
        same(got, S.verify(t, draft, d, u))


@pytest.mark.parametrize("cols", [7, 70000])
@pytest.mark.parametrize("temperature", [1e-307, 1e-40, 1e40, 1e307])
def test_extreme_temperatures(layers, temperature, cols):
    """All to the largest score, or to all that are not masked alike."""
    t, q, d, u = case(4, 2, cols, torch.float32, cols)
    t[:, :, ::3], q[:, :, ::3] = -math.inf, -math.inf
    u[:] = (u * 64).floor() / 64 + 1 / 128  # (off the borders of equal shares)
    got = layers.verify_drafts(t, None, d, u, temperature=temperature)
    same(got, S.verify(t, None, d, u, temperature=temperature))
    got = layers.verify_drafts(t, q, d, u, temperature=temperature)
    want = S.verify(t, q, d, u, temperature=temperature)
    # (of shares that are alike, nothing or a rounding is left of the difference)
    stood = torch.arange(3) < want[1][:, None]
    assert torch.equal(got.accepted.cpu(), want[1])
    assert torch.equal(got.outcomes.cpu()[stood], want[0][stood])
    assert torch.isfinite(t.flatten(0, 1).cpu()[
        torch.arange(4) * 3 + got.accepted.cpu(),
        got.outcomes.cpu()[torch.arange(4), got.accepted.cpu()]]).all()


@pytest.mark.parametrize("cols", [6, 4000, 9001, 70000])
@pytest.mark.parametrize("kind", ["logits", "weights"])
def test_rows_without_outcomes(layers, kind, cols):
    t, q, d, u = case(9, 2, cols, torch.float32, 7, kind)
    gone = -math.inf if kind == "logits" else 0.0
    t[0, 0], q[1, 0], t[2], q[2] = gone, gone, gone, gone
    t[3, 0, 3], q[4, 0, 4] = math.nan, math.nan
    t[5, 0, 1], q[6, 0, 2] = math.inf, math.inf
    t[7, 0, :cols - 1], t[8, 0, 1:] = gone, gone
    got = layers.verify_drafts(t, q, d, u, kind)
    same(got, S.verify(t, q, d, u, kind))
    assert got.outcomes[[0, 2, 3, 5], 0].tolist() == [-1] * 4
    assert (got.outcomes[[1, 4, 6], 0] >= 0).all() and got.accepted[[0, 1, 2, 3, 4, 5, 6]].eq(0).all()


def test_masks(layers):
    """Outcomes ruled out never come; rows of the type's lowest number are uniform."""
    n, k, cols = 200, 2, 3000
    t, q, d, u = case(n, k, cols, torch.bfloat16, 9)
    out = torch.rand(cols, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.5
    out[d.unique()] = False
    t[..., out], q[..., out] = -math.inf, -math.inf
    got = layers.verify_drafts(t, q, d, u)
    same(got, S.verify(t, q, d, u))
    come = got.outcomes[got.outcomes >= 0]
    assert not out[come].any()
    for dtype in TYPES:
        low = torch.full((50, 1, 1000), torch.finfo(dtype).min, dtype=dtype, device=DEV)
        got = layers.verify_drafts(low, None, d[:50, :0], u[:50, :1])
        assert torch.equal(got.outcomes[:, 0], (u[:50, 0] * 1000).long())


def test_weights_of_any_scale(layers):
    t, q, d, u = case(20, 3, 700, torch.float32, 11, "weights")
    want = S.verify(t, q, d, u, "weights")
    same(layers.verify_drafts(t, q, d, u, "weights"), want)
    # powers of two: the same numbers
    same(layers.verify_drafts(t * 2.0 ** 120, q * 2.0 ** -60, d, u, "weights"), want)


@pytest.mark.parametrize("cols", [3, 1000, 60000])
@pytest.mark.parametrize("drafts", [1, 40])
def test_nothing_left_of_the_difference(layers, cols, drafts):
    """A draft that is refused although the target's probabilities are nowhere above it: drawn from
    the target, whose only two outcomes are alike."""
    t = torch.zeros((2, drafts + 1, cols), device=DEV)
    t[:, :, 0] = t[:, :, cols - 2] = 0.5
    d = torch.full((2, drafts), cols - 1, device=DEV)
    u = torch.zeros((2, drafts + 1), device=DEV)
    u[:, -1] = torch.tensor([0.25, 0.75])
    got = layers.verify_drafts(t, t[:, :drafts], d, u, "weights")
    assert got.accepted.tolist() == [0, 0]
    assert got.outcomes[:, 0].tolist() == [0, cols - 2] and (got.outcomes[:, 1:] == -1).all()


def test_distributed_as_the_target(layers):
    """However far off the draft is, the first outcome is the target's.  Counts of N draws lie
    within 6 of their standard deviations (a chance of 2e-9 each not to)."""
    n, cols = 40000, 7
    g = torch.Generator().manual_seed(3)
    t, q = torch.randn(2, cols, generator=g) * 1.5, torch.randn(1, cols, generator=g) * 1.5
    d = torch.multinomial(torch.softmax(q[0], 0), n, True, generator=g)[:, None].to(DEV)
    u = torch.rand((n, 2), generator=g, dtype=torch.float64).to(DEV)
    got = layers.verify_drafts(t.to(DEV).expand(n, 2, cols), q.to(DEV).expand(n, 1, cols), d, u)
    p = torch.softmax(t[0].double(), 0)
    count = torch.bincount(got.outcomes[:, 0].cpu(), minlength=cols)
    assert ((count - n * p).abs() <= 6 * torch.sqrt(n * p * (1 - p))).all()
    both = got.outcomes[got.accepted == 1, 1].cpu()
    p, m = torch.softmax(t[1].double(), 0), len(both)
    count = torch.bincount(both, minlength=cols)
    assert ((count - m * p).abs() <= 6 * torch.sqrt(m * p * (1 - p))).all()


def test_shapes_strides_and_types(layers):
    t, q, d, u = case(12, 3, 130, torch.bfloat16, 13)
    want = layers.verify_drafts(t, q, d, u)
    got = layers.verify_drafts(t.reshape(3, 4, 4, 130), q.reshape(3, 4, 3, 130),
                               d.reshape(3, 4, 3), u.reshape(3, 4, 4))
    assert got.outcomes.shape == (3, 4, 4) and got.accepted.shape == (3, 4)
    assert torch.equal(got.outcomes.reshape(12, 4), want.outcomes)
    one = layers.verify_drafts(t[0], q[0], d[0], u[0])
    assert one.outcomes.shape == (4,) and one.accepted.shape == ()
    assert torch.equal(one.outcomes, want.outcomes[0])
    # rows out of a wider table, drafts and numbers by columns
    wide = torch.full((12, 4, 201), math.nan, dtype=torch.bfloat16, device=DEV)
    wide[..., 3:133] = t
    again = layers.verify_drafts(wide[..., 3:133], q, d.T.contiguous().T, u.T.contiguous().T)
    assert torch.equal(again.outcomes, want.outcomes)
    # 32-bit numbers stand for themselves
    got = layers.verify_drafts(t, q, d, u.float())
    assert torch.equal(got.outcomes, layers.verify_drafts(t, q, d, u.float().double()).outcomes)
    for n, k in ((0, 0), (0, 3)):
        empty = layers.verify_drafts(t[:n, :k + 1], q[:n, :k], d[:n, :k], u[:n, :k + 1])
        assert empty.outcomes.shape == (n, k + 1) and empty.accepted.shape == (n,)


def test_refusals(layers):
    t, q, d, u = case(4, 2, 30, torch.float32, 15)
    f = layers.verify_drafts
    bad = [
        lambda: f(t, q, d, u, "scores"), lambda: f(t, q, d, u, "logits", 0.0),
        lambda: f(t, q, d, u, "logits", math.nan), lambda: f(t, q, d, u, "logits", 5e-324),
        lambda: f(t, q, d, u, "weights", 2.0), lambda: f(t[:, :2], q, d, u),
        lambda: f(t, q[:, :1], d, u), lambda: f(t, q.half(), d, u), lambda: f(t, q, d[:, :1], u),
        lambda: f(t, q, d.int(), u), lambda: f(t, q, d, u[:, :2]), lambda: f(t, q, d, u.half()),
        lambda: f(t, q, d.cpu(), u), lambda: f(t, q, d, u.cpu()), lambda: f(t.cpu(), q, d, u),
        lambda: f(t.double(), q.double(), d, u), lambda: f(t[0, 0], None, d[0, :0], u[0, :1]),
        lambda: f(t[:, :, :0], q[:, :, :0], d, u), lambda: f(t[:, :0], None, d[:, :0], u[:, :0]),
        lambda: f(t.transpose(1, 2), None, d, u),
        lambda: f(t.detach().clone().requires_grad_(True), q, d, u),
        lambda: f(t, q.detach().clone().requires_grad_(True), d, u),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was let through")


def test_streams_and_graphs(layers):
    """On another stream, and captured: two graphs replayed in turn with eager calls between."""
    cases = [case(3, 4, 6000, torch.float32, 20), case(30, 2, 900, torch.bfloat16, 21)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = layers.verify_drafts(*cases[0])
    torch.cuda.current_stream().wait_stream(s)
    same(other, S.verify(*cases[0]))
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layers.verify_drafts(*c)
        graphs.append((g, c, out))
    for k in range(3):
        for (g, c, out), fresh in zip(graphs, (case(3, 4, 6000, torch.float32, 30 + k),
                                               case(30, 2, 900, torch.bfloat16, 40 + k))):
            for a, b in zip(c, fresh):
                a.copy_(b)
            g.replay()
            torch.cuda.synchronize()
            same(out, S.verify(*c))


def test_head_in_integers_and_its_answers(layers):
    """Features of every position through norm and 8-bit layers to logits, which verify what a
    narrower head drafted."""
    g = torch.Generator().manual_seed(17)
    n, k, width, cols = 6, 3, 96, 700

    def table(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)

    x, w1, w2 = table(n, k + 1, width), table(2 * width, width) / 10, table(cols, 2 * width) / 10
    b1, b2, small = table(2 * width) / 3, table(cols) / 3, table(cols, width) / 10
    h = layers.linear_quantized(layers.layer_norm(x), layers.quantize(w1), b1, "gelu")
    logits = layers.linear_quantized(h, layers.quantize(w2), b2)
    assert logits.shape == (n, k + 1, cols)
    draft = layers.linear(layers.layer_norm(x[:, :k].contiguous()), small)
    d = layers.log_probs(draft, top=1).top_index[..., 0]
    u = torch.rand((n, k + 1), generator=g, dtype=torch.float64).to(DEV)
    same(layers.verify_drafts(logits, draft, d, u), S.verify(logits, draft, d, u))
    same(layers.verify_drafts(logits, None, d, u), S.verify(logits, None, d, u))
    v = layers.verify_drafts(logits, draft, d, u)
    scored = layers.log_probs(logits, v.outcomes)
    assert torch.isfinite(scored.logp).all()


def test_long_scores(layers):
    """More than 2^32 bytes of scores: the last sequences' answers are those of a call of theirs."""
    g = torch.Generator(device=DEV).manual_seed(12)
    n, k, cols = 5000, 7, 60001
    t = torch.randn((n, k + 1, cols), generator=g, device=DEV, dtype=torch.float16)
    q = torch.randn((n, k, cols), generator=g, device=DEV, dtype=torch.float16)
    q[:, :5] = t[:, :5]
    d = torch.randint(0, cols, (n, k), generator=g, device=DEV)
    u = torch.rand((n, k + 1), generator=g, device=DEV, dtype=torch.float64)
    got = layers.verify_drafts(t, q, d, u)
    assert (got.accepted >= 5).all()
    want = layers.verify_drafts(t[-5:], q[-5:], d[-5:], u[-5:])
    same(layers.Verified(got.outcomes[-5:], got.accepted[-5:]),
         (want.outcomes.cpu(), want.accepted.cpu()))
