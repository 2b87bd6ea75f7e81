"""Plain 64-bit forms of the layers and error bounds of a 32-bit computation of them.

Bounds: u = 2^-24 is the unit roundoff of fp32, v that of the element type.  A result carries
v |result| for its rounding to the type (plus half the type's smallest step), and n u sum|terms|
for a sum of n terms in any order; a chain of a few operations is counted as 16 u of what it
passes through.  exp and log of the device are within a few ulp.
"""
import math

import torch

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def d(t):
    return None if t is None else t.detach().cpu().double()


def check(got, want, bound, dtype, what):
    got = d(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    err = (got - want).abs()
    limit = ROUND[dtype] * want.abs() + TINY[dtype] + bound
    bad = ~(same | (err <= limit))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst "
                           f"{float(err[bad].max())} against {float(limit.expand_as(err)[bad].min())}")


# ------------------------------------------------------------------ layer norm

def norm(x, w, b, eps):
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    h = (x - mean) * rstd
    return h * (1 if w is None else w) + (0 if b is None else b), h, rstd


def norm_bound(x, w, b, eps):
    # h is off by what the mean is (log-depth sums: 64 u max|x|), times rstd, and relative to
    # itself by rstd's own error
    _, h, rstd = norm(x, w, b, eps)
    dh = 64 * U * (rstd * x.abs().amax(-1, keepdim=True) + h.abs())
    return dh * (1 if w is None else w.abs()) + 16 * U * (0 if b is None else b.abs()), dh


def norm_grads(x, w, eps, dy):
    n = x.shape[-1]
    _, h, rstd = norm(x, w, None, eps)
    g = dy * (1 if w is None else w)
    c1, c2 = g.sum(-1, keepdim=True) / n, (g * h).sum(-1, keepdim=True) / n
    return rstd * (g - c1 - h * c2), (dy * h).sum(0), dy.sum(0)


def norm_grad_bounds(x, w, eps, dy):
    _, h, rstd = norm(x, w, None, eps)
    _, dh = norm_bound(x, w, None, eps)
    g = (dy * (1 if w is None else w)).abs()
    mg, mgh = g.mean(-1, keepdim=True), (g * h.abs()).mean(-1, keepdim=True)
    e2 = (g * dh).mean(-1, keepdim=True)
    dx = rstd * (64 * U * (g + mg + h.abs() * mgh) + dh * mgh + h.abs() * e2)
    # rstd's own relative error
    dx = dx + 64 * U * rstd * (g + mg + h.abs() * mgh) * (1 + rstd * x.abs().amax(-1, keepdim=True))
    rows = x.shape[0]
    dw = (rows + 16) * U * (dy * h).abs().sum(0) + (dy.abs() * dh).sum(0)
    return dx, dw, (rows + 16) * U * dy.abs().sum(0)


# ------------------------------------------------------------------ linear

def act(name, z):
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if name == "tanh":
        return torch.tanh(z), 1 - torch.tanh(z) ** 2
    return z, torch.ones_like(z)


# Lipschitz constants of a and a'; relu's slope is taken at sums that fp32 has exactly
LIP = {"none": (1, 0), "relu": (1, 0), "gelu": (1.13, 0.8), "silu": (1.1, 0.5), "tanh": (1, 0.77)}


def linear(x, w, b, name, r):
    z = x @ w.T + (0 if b is None else b)
    y, slope = act(name, z)
    return y + (0 if r is None else r), z, slope


def linear_bounds(x, w, b, name, r):
    k = x.shape[-1]
    y, z, _ = linear(x, w, b, name, r)
    ez = (k + 16) * U * (x.abs() @ w.abs().T + (0 if b is None else b.abs()))
    return LIP[name][0] * ez + 16 * U * (z.abs() + (0 if r is None else r.abs())), ez


def linear_grads(x, w, b, name, dy):
    dz = dy * linear(x, w, b, name, None)[2]
    return dz @ w, dz.T @ x, dz.sum(0)


def linear_grad_bounds(x, w, b, name, dy, dtype, rounded=True):
    rows, n_out = dy.shape
    dz = (dy * linear(x, w, b, name, None)[2]).abs()
    ez = linear_bounds(x, w, b, name, None)[1]
    e = 0 if name == "none" else dy.abs() * (LIP[name][1] * ez + 32 * U)
    # dz enters the products rounded to the type (unless it is small)
    er = e + (0 if name == "none" or not rounded else ROUND[dtype] * dz + TINY[dtype])
    full = dz + er
    dx = er @ w.abs() if name != "none" else 0
    dw = er.T @ x.abs() if name != "none" else 0
    return (dx + (n_out + 16) * U * (full @ w.abs()), dw + (rows + 16) * U * (full.T @ x.abs()),
            (e.sum(0) if name != "none" else 0) + (rows + 16) * U * dz.sum(0))


# ------------------------------------------------------------------ scores

def scores(z, t, top, kind, temperature):
    """logp [rows, n], entropy, top_logp, top_index, and (p, log p) for the gradient."""
    if kind == "weights":
        total = z.sum(-1, keepdim=True)
        empty = total == 0
        p = torch.where(empty, 0.0, z / total)
        lp = torch.where(empty, -math.inf, torch.log(z) - torch.log(total))
    else:
        s = z / temperature
        m = s.amax(-1, keepdim=True)
        empty = m == -math.inf
        e = torch.exp(s - torch.where(empty, 0.0, m))
        total = e.sum(-1, keepdim=True)
        p = torch.where(empty, 0.0, e / total)
        lp = torch.where(empty, -math.inf, s - m - torch.log(total))
    h = -torch.where(p == 0, 0.0, p * lp).sum(-1)
    logp = lp.gather(-1, t.clamp(0, z.shape[-1] - 1))
    logp = torch.where(t == -1, 0.0, logp)
    logp = torch.where((t < -1) | (t >= z.shape[-1]), math.nan, logp)
    order = torch.sort(z, dim=-1, descending=True, stable=True)[1][:, :top]
    return logp, h, lp.gather(-1, order), order, p, lp


def score_bounds(z, kind, temperature):
    """Bounds of a log probability (per outcome) and of the entropy."""
    n = z.shape[-1]
    _, h, _, _, p, lp = scores(z, torch.zeros((z.shape[0], 0), dtype=torch.int64), 0, kind,
                               temperature)
    finite = torch.where(p > 0, lp, 0.0).abs()
    # a sum of n terms in fp32, each an exp of a number of |d| (its argument rounded twice);
    # |d| <= |log p| + log n
    span = finite + math.log(max(n, 2))
    ds = (n + 64) * U + 8 * U * (p * span).sum(-1, keepdim=True)
    if kind == "weights":
        # every log w is off by a few ulp, of at most ln of the weights' range (-87 .. 87)
        span = span + 90
    dlp = ds + 8 * U * span
    dh = (ds * (1 + h.abs().unsqueeze(-1)) + (n + 64) * U * (p * span).sum(-1, keepdim=True) * 2
          + 8 * U * (p * span * span).sum(-1, keepdim=True)).squeeze(-1)
    return dlp, dh


def score_grad(z, t, temperature, g, gh):
    _, h, _, _, p, lp = scores(z, t, 0, "logits", temperature)
    n = z.shape[-1]
    ok = (t >= 0) & (t < n)
    g = torch.where(ok, g, 0.0)
    empty = (z == -math.inf).all(-1, keepdim=True)
    picked = torch.zeros_like(z).scatter_add_(-1, t.clamp(0, n - 1), g)
    plp = torch.where(p == 0, 0.0, p * lp)
    dz = picked - p * g.sum(-1, keepdim=True) - gh[:, None] * (plp + p * h[:, None])
    return torch.where(empty, 0.0, dz / temperature)


def score_grad_bound(z, t, temperature, g, gh):
    _, h, _, _, p, lp = scores(z, t, 0, "logits", temperature)
    dlp, dh = score_bounds(z, "logits", temperature)
    n = z.shape[-1]
    ok = (t >= 0) & (t < n)
    ga = torch.where(ok, g.abs(), 0.0)
    all_g = ga.sum(-1, keepdim=True)
    alp = torch.where(p == 0, 0.0, lp.abs())
    size = all_g + gh.abs()[:, None] * (alp + h[:, None])
    picked = torch.zeros_like(z).scatter_add_(-1, t.clamp(0, n - 1), ga)
    shots = t.shape[-1]
    e = p * (dlp + 16 * U) * size + p * gh.abs()[:, None] * (dlp + dh[:, None])
    e = e + (shots + 16) * U * (picked + p * all_g)
    return e / temperature
