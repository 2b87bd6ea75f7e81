"""Drafts verified by several workgroups to a sequence, in both forms: rows behind a refused draft
read, or passed over.  test_verify_ways_cpu.py holds the sizes to the form they are for."""
import math

import pytest
import torch

from tests import serving_oracle as S
from tests.test_gpu_layers import DEV, TYPES
from tests.test_gpu_verify import case, layers, same  # noqa: F401 (layers: a fixture)

pytestmark = pytest.mark.gpu

INT32_MAX = 2 ** 31 - 1

SHORT = (6, 70, 7)  # 16-bit rows shorter than a pack
# the form with the draft's scores, and with drafts that were certain
LONG = {(8, 12, 4000): ("passed", "passed"), (9, 70, 300): ("passed", "passed"),
        SHORT: ("passed", "passed"), (70, 5, 30001): ("passed", "read"),
        (8, 3, 70000): ("read", "read"), (9, 9, 20001): ("read", "read"),
        (300, 5, 6000): ("read", "read")}
GRAPHS = {(4, 12, 5000): "passed", (3, 70, 900): "passed", (3, 4, 60000): "read"}
SIZES = pytest.mark.parametrize("n,k,cols", list(LONG))
KINDS = pytest.mark.parametrize("kind", ["logits", "weights"])


def ends(n, k):
    """Where the n sequences' drafts are made to end: everywhere, k (not at all) among them."""
    return torch.arange(n) * 7 % (k + 1)


def alike(n, k, cols, dtype, seed, kind="logits"):
    """A draft that is the target: every drafted outcome stands."""
    t, q, d, u = case(n, k, cols, dtype, seed, kind)
    q.copy_(t[:, :k])
    return t, q, d, u


@KINDS
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@SIZES
def test_verify(layers, n, k, cols, dtype, kind):
    t, q, d, u = case(n, k, cols, dtype, n + k + cols, kind, near=0.05)
    for draft in (q, None):
        same(layers.verify_drafts(t, draft, d, u, kind), S.verify(t, draft, d, u, kind))


@KINDS
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@SIZES
def test_drafts_that_end_early(layers, n, k, cols, dtype, kind):
    """-1 and any other index outside the row ends the drafts; what is behind is not looked at, nor is
    the draft's row there."""
    t, q, d, u = alike(n, k, cols, dtype, 5, kind)
    end = ends(n, k)
    for s in range(n):
        if end[s] < k:
            d[s, end[s]] = (-1, cols, -(2 ** 63), 2 ** 63 - 1)[s % 4]
            q[s, end[s]:] = math.nan
            t[s, end[s] + 1:] = math.nan
    got = layers.verify_drafts(t, q, d, u, kind)
    assert torch.equal(got.accepted.cpu(), end)
    same(got, S.verify(t, q, d, u, kind))
    assert (got.outcomes.cpu()[torch.arange(n), end] >= 0).all()
    # certain drafts: uniform numbers of 0 accept whatever has a share
    u[:, :k] = 0
    got = layers.verify_drafts(t, None, d, u, kind)
    assert torch.equal(got.accepted.cpu(), end)
    same(got, S.verify(t, None, d, u, kind))
    # none at all
    d[:] = -1
    got = layers.verify_drafts(t, q, d, u, kind)
    assert got.accepted.eq(0).all()
    same(got, S.verify(t, q, d, u, kind))


@pytest.mark.parametrize("mask", [-math.inf, "lowest"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@SIZES
def test_drafts_without_a_share(layers, mask, dtype, n, k, cols):
    """A uniform number of 0 accepts whatever has a share, and nothing that has none."""
    mask = torch.finfo(dtype).min if mask == "lowest" else mask
    t, q, d, u = case(n, k, cols, dtype, n + k + cols)
    u[:, :k] = 0
    end = ends(n, k)
    for s in range(n):
        if end[s] < k:
            t[s, end[s], d[s, end[s]]] = mask
            if s % 2:  # nor of the draft's
                q[s, end[s], d[s, end[s]]] = mask
    for draft in (q, None):
        got = layers.verify_drafts(t, draft, d, u)
        assert torch.equal(got.accepted.cpu(), end)
        same(got, S.verify(t, draft, d, u))


@KINDS
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16], ids=str)
@SIZES
def test_rows_without_outcomes(layers, n, k, cols, dtype, kind):
    """Behind accepted drafts: rows of the target, of the draft or of both with nothing left, a NaN or
    an infinity, in turn."""
    gone = -math.inf if kind == "logits" else 0.0
    t, q, d, u = alike(n, k, cols, dtype, 7, kind)
    end = ends(n, k)
    none = torch.zeros(n, dtype=torch.bool)
    for s in range(n):
        i, way = int(end[s]), s % 7
        if i == k:  # the row behind the drafts
            t[s, i] = gone if way % 2 else math.nan
            none[s] = True
            continue
        rows = {0: (t,), 1: (q,), 2: (t, q), 3: (t,), 4: (q,), 5: (t,), 6: (q,)}[way]
        for r in rows:
            if way < 3:
                r[s, i] = gone
            else:
                r[s, i, (3 * s + 1) % cols] = math.nan if way < 5 else math.inf
        none[s] = any(r is t for r in rows)
    got = layers.verify_drafts(t, q, d, u, kind)
    assert torch.equal(got.accepted.cpu(), end)
    same(got, S.verify(t, q, d, u, kind))
    drawn = got.outcomes.cpu()[torch.arange(n), end]
    assert torch.equal(drawn < 0, none)


@SIZES
def test_nothing_left_of_the_difference(layers, n, k, cols):
    """Refused although the target's probabilities are nowhere above the draft's, behind drafts that
    stand: drawn from the target, whose only two outcomes are alike."""
    t = torch.zeros((n, k + 1, cols), device=DEV)
    t[:, :, 0] = t[:, :, cols - 2] = 0.5
    d = torch.zeros((n, k), dtype=torch.int64, device=DEV)
    end = ends(n, k)
    for s in range(n):
        d[s, end[s]:] = cols - 1
    u = torch.full((n, k + 1), 0.5, device=DEV)
    u[:, -1] = torch.tensor([0.25, 0.75], device=DEV).repeat(n)[:n]
    got = layers.verify_drafts(t, t[:, :k], d, u, "weights")
    assert torch.equal(got.accepted.cpu(), end)
    drawn = got.outcomes.cpu()[torch.arange(n), end]
    assert drawn.tolist() == [0 if s % 2 == 0 else cols - 2 for s in range(n)]
    for s in range(n):
        assert got.outcomes[s, :end[s]].eq(0).all() and got.outcomes[s, end[s] + 1:].eq(-1).all()


@SIZES
def test_rows_out_of_wider_tables(layers, n, k, cols):
    t, q, d, u = case(n, k, cols, torch.float16, 13)
    want = layers.verify_drafts(t, q, d, u)
    wt = torch.full((n, k + 1, cols + 9), math.nan, dtype=torch.float16, device=DEV)
    wq = torch.full((n, k, cols + 5), math.nan, dtype=torch.float16, device=DEV)
    wt[..., 3:cols + 3], wq[..., 1:cols + 1] = t, q
    got = layers.verify_drafts(wt[..., 3:cols + 3], wq[..., 1:cols + 1], d, u)
    assert torch.equal(got.outcomes, want.outcomes) and torch.equal(got.accepted, want.accepted)


def test_graphs(layers):
    """Every form captured, replayed in turn on new numbers with eager calls between: counters that a
    replay leaves behind are not the next one's."""
    cases = [case(*s, torch.bfloat16, 20 + i) for i, s in enumerate(GRAPHS)]
    graphs = []
    for c in cases:
        for draft in (c[1], None):
            args = (c[0], draft, c[2], c[3])
            layers.verify_drafts(*args)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = layers.verify_drafts(*args)
            graphs.append((g, args, out))
    for r in range(4):
        for i, (size, c) in enumerate(zip(GRAPHS, cases)):
            for a, b in zip(c, case(*size, torch.bfloat16, 100 + 10 * r + i, near=(0.0, 0.7)[r % 2])):
                a.copy_(b)
        for g, args, out in graphs:
            g.replay()
            eager = layers.verify_drafts(*args)
            torch.cuda.synchronize()
            want = S.verify(*args)
            same(out, want)
            same(eager, want)


def test_two_streams_at_once(layers):
    """Calls of every form in flight on two streams: each has its own workspace."""
    cases = [case(*s, torch.float16, 40 + i) for i, s in enumerate(GRAPHS)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for c in cases:
            for s in streams:
                with torch.cuda.stream(s):
                    got.append((c, layers.verify_drafts(*c)))
    torch.cuda.synchronize()
    wants = [S.verify(*c) for c in cases]
    for c, v in got:
        same(v, wants[[x is c for x in cases].index(True)])


@pytest.mark.parametrize("n,k,cols,kind", [(4200000, 0, 4, "logits"), (4200000, 1, 3, "weights"),
                                           (120000, 70, 5, "logits")])
def test_more_sequences_than_a_grid_holds(layers, n, k, cols, kind):
    """Answers of the whole are those of calls of its parts, which reach both sides of where one
    launch ends: 4194303 sequences of a workgroup each, 8388607 workgroups of rows."""
    g = torch.Generator(device=DEV).manual_seed(n + k)
    t = torch.randn((n, k + 1, cols), generator=g, device=DEV)
    q = t[:, :k] + 0.1 * torch.randn((n, k, cols), generator=g, device=DEV)
    if kind == "weights":
        t, q = t.exp(), q.exp()
    t, q = t.half(), q.half()
    d = torch.randint(-1 if k > 1 else 0, cols, (n, k), generator=g, device=DEV)
    u = torch.rand((n, k + 1), generator=g, device=DEV, dtype=torch.float64)
    u[:, :k] *= u[:, :k]
    for draft in (q, None):
        got = layers.verify_drafts(t, draft, d, u, kind)
        assert (got.outcomes.gather(1, got.accepted[:, None]) >= 0).all()
        size = 50000 if k > 1 else 2100000
        for a in range(0, n, size):
            b = min(n, a + size)
            want = layers.verify_drafts(t[a:b], None if draft is None else draft[a:b], d[a:b],
                                        u[a:b], kind)
            assert torch.equal(got.outcomes[a:b], want.outcomes)
            assert torch.equal(got.accepted[a:b], want.accepted)
        for a in (0, (INT32_MAX // 512 if k < 2 else n // 2) - 20, n - 40):
            part = slice(a, a + 40)
            args = (t[part], None if draft is None else draft[part], d[part], u[part], kind)
            same(layers.Verified(got.outcomes[part], got.accepted[part]), S.verify(*args))
