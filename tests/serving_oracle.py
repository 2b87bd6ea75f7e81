"""Plain 64-bit forms of rows in 8-bit integers, of linear layers on them and of the verification of
drafted outcomes.

Bounds of the linear layers (u = 2^-24): the sum of integers is exact, its rounding and the two
steps' products are 3 u |z|, the bias one more u of what it gives; a chain of a few operations
behind that is counted as 16 u of what it passes through, as in layers_oracle.
"""
import math

import torch

from tests import layers_oracle as O


def quantized(x):
    """(integers, scales): 127 x / a is one division of exact numbers, so that a tie is one."""
    x = O.d(x)
    if x.shape[-1] == 0:
        return x.to(torch.int8), torch.zeros(x.shape[:-1])
    most = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(x).all(-1, keepdim=True)
    q = torch.round(127 * x / torch.where(finite & (most > 0), most, 1.0))
    scales = torch.where(finite, most, math.nan).float() / 127
    return torch.where(finite, q, 0.0).to(torch.int8), scales.squeeze(-1)


def products(xq, wq):
    """Sums of integers: below 2^53 in any order."""
    return xq.cpu().double() @ wq.cpu().double().T


def linear(xq, xs, wq, ws, b, name, r):
    """(y, bound) of the integers and their steps."""
    z = products(xq, wq) * O.d(xs)[:, None] * O.d(ws)
    ez = 4 * O.U * (z.abs() + (0 if b is None else (z + b).abs()))
    z = z + (0 if b is None else b)
    y = O.act(name, z)[0]
    bound = O.LIP[name][0] * ez + 16 * O.U * (z.abs() + (0 if r is None else r.abs()))
    return y + (0 if r is None else r), bound


def probabilities(row, kind, temperature):
    """None where the row has no outcomes."""
    row = O.d(row)
    if kind == "logits":
        m = row.max()
        if not math.isfinite(m) or row.isnan().any():
            return None
        row = torch.exp((row - m) / temperature)
    total = row.sum()
    if not (math.isfinite(total) and total > 0):
        return None
    return row / total


def drawn(weights, u):
    sums = weights.cumsum(0)
    over = (sums > u * sums[-1]).nonzero()
    if len(over):
        return int(over[0])
    return int((weights > 0).nonzero()[-1])


def verify(target, draft, drafted, uniforms, kind="logits", temperature=1.0):
    """(outcomes, accepted) of [sequences, drafts + 1, outcomes] one after the other."""
    n, rows, cols = target.shape
    outcomes = torch.full((n, rows), -1, dtype=torch.int64)
    accepted = torch.zeros(n, dtype=torch.int64)
    u = uniforms.detach().cpu().double()
    for s in range(n):
        for i in range(rows):
            p = probabilities(target[s, i], kind, temperature)
            d = int(drafted[s, i]) if i + 1 < rows else -1
            rest = p
            if 0 <= d < cols:
                if draft is None:
                    q = torch.zeros(cols, dtype=torch.float64)
                    q[d] = 1
                else:
                    q = probabilities(draft[s, i], kind, temperature)
                if p is not None and q is not None and float(u[s, i] * q[d]) < float(p[d]):
                    outcomes[s, i] = d
                    accepted[s] += 1
                    continue
                if p is not None and q is not None and ((p - q) > 0).any():
                    rest = (p - q).clamp(min=0)
            if rest is not None:
                outcomes[s, i] = drawn(rest, float(u[s, -1]))
            break
    return outcomes, accepted
