"""The layers around a circuit, as a hybrid model calls them: layer norm of the features, the
linear layers that turn features into angles and read-outs into logits, and the scores of given
outcomes (log probabilities, entropy, most probable alternatives) from logits or from the
circuit's own outcome probabilities.

A case names an operator with its sizes, element type and direction; `train` adds the gradients
of every input for a given cotangent.  In the plain form everything is computed in 32 bits by
elementary torch operations and rounded once; with `own` set the calls are those of
paper_2607_11985_amd.layers.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-5
# bounds of the drawn cases: elements, products and scores of the largest listed ones
_MOST_NORM = 8192 * 4096
_MOST_LINEAR = 8192 * 4096 * 4096
_MOST_SCORES = 4096 * 32768


def _norm(rows, cols, dtype, train, pad=0):
    return {"op": "layer_norm", "rows": rows, "cols": cols, "dtype": dtype, "train": train,
            "pad": pad}


def _linear(rows, n_in, n_out, dtype, train, act="none", residual=False, pad=0):
    return {"op": "linear", "rows": rows, "in": n_in, "out": n_out, "dtype": dtype,
            "train": train, "act": act, "residual": residual, "pad": pad}


def _scores(rows, cols, dtype, train, kind="logits", shots=1, top=0, masked=0.0):
    return {"op": "log_probs", "rows": rows, "cols": cols, "dtype": dtype, "train": train,
            "kind": kind, "shots": shots, "top": top, "masked": masked}


def listed():
    return [
        # 64 samples' 16 features before the angle encoding: latency
        dict(_norm(64, 16, "f32", False), name="norm_f32_64x16"),
        # features of an odd width out of a wider table, in training
        dict(_norm(1000, 769, "f32", True, pad=7), name="norm_train_f32_1000x769"),
        # a large batch of wide features in training
        dict(_norm(8192, 4096, "bf16", True), name="norm_train_bf16_8192x4096"),
        # 16 expectations to 10 logits, the smallest read-out: latency
        dict(_linear(64, 16, 10, "f32", False), name="linear_f32_64x16x10"),
        # one sample's wide features through a square layer with its residual: serving
        dict(_linear(1, 4096, 4096, "bf16", False, "gelu", True),
             name="linear_bf16_1x4096x4096"),
        # features to the 384 per-sample angles of a 16-qubit, 8-layer circuit, in training
        dict(_linear(1024, 768, 384, "f32", True, "tanh"), name="linear_train_f32_1024x768x384"),
        # the 2^14 outcome probabilities of a batch read out into classes: a long sum, few
        # outputs, odd sizes
        dict(_linear(301, 16384, 101, "f16", True), name="linear_train_f16_301x16384x101"),
        # a wide layer over a large batch in training: the most arithmetic of all
        dict(_linear(8192, 4096, 4096, "bf16", True, "gelu", True),
             name="linear_train_bf16_8192x4096x4096"),
        # a small classifier's loss in training: latency
        dict(_scores(64, 10, "f32", True), name="scores_train_f32_64x10"),
        # 1024 measured shots of each of 256 states of 16 qubits, the likeliest outcomes too
        dict(_scores(256, 65536, "f32", False, "weights", shots=1024, top=8),
             name="scores_weights_f32_256x65536"),
        # one state of 20 qubits: a single long row
        dict(_scores(1, 1 << 20, "f32", False, "weights", shots=100, top=16),
             name="scores_weights_f32_1x1048576"),
        # logits over many outcomes, some of them ruled out, in training
        dict(_scores(4096, 32768, "bf16", True, top=5, masked=0.1),
             name="scores_train_bf16_4096x32768"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["layer_norm", "linear", "linear", "log_probs"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        train = rng.random() < 0.6
        pad = rng.choice([0, 0, 1, 8])
        if op == "layer_norm":
            # from 4 columns on: with 2 the gradient is what eps leaves of a cancellation
            case = _norm(log_int(1, 16384), log_int(4, 16384), dtype, train, pad)
            if case["rows"] * case["cols"] <= _MOST_NORM:
                return case
        elif op == "linear":
            # relu's slope at a sum whose sign is its last bit's cannot be compared in 32 bits
            acts = ["none", "gelu", "silu", "tanh"] + (["relu"] if dtype != "f32" else [])
            case = _linear(log_int(1, 8192), log_int(1, 16384), log_int(1, 16384), dtype, train,
                           rng.choice(acts), rng.random() < 0.5, pad)
            # 32-bit products run at a sixteenth of the 16-bit rate
            most = _MOST_LINEAR // (16 if dtype == "f32" else 1)
            if case["rows"] * case["in"] * case["out"] <= most:
                return case
        else:
            kind = rng.choice(["logits", "logits", "weights"])
            cols = 1 << rng.randint(4, 20) if kind == "weights" else log_int(2, 1 << 18)
            case = _scores(log_int(1, 8192), cols, "f32" if kind == "weights" else dtype,
                           train and kind == "logits", kind,
                           log_int(1, 1024) if kind == "weights" else 1,
                           min(rng.choice([0, 1, 5, 20]), cols),
                           rng.choice([0.0, 0.3]) if kind == "logits" else 0.0)
            if case["rows"] * case["cols"] <= _MOST_SCORES:
                return case


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _table(g, rows, cols, pad, dtype, scale=1.0):
    """rows x cols out of a table whose rows are `pad` elements longer."""
    t = torch.randn((rows, cols + pad), generator=g, device="cuda") * scale
    return t.to(dtype)[:, :cols]


def prepare(case, seed):
    g, dtype, op = _generator(seed), _TYPES[case["dtype"]], case["op"]
    rows = case["rows"]
    state = {"case": case, "dtype": dtype}
    if op == "layer_norm":
        cols = case["cols"]
        # rows of unlike level and spread
        x = torch.randn((rows, cols + case["pad"]), generator=g, device="cuda")
        x *= torch.rand((rows, 1), generator=g, device="cuda") * 2 + 0.5
        x += torch.randn((rows, 1), generator=g, device="cuda")
        state["x"] = x.to(dtype)[:, :cols]
        state["w"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
        state["b"] = (0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
        state["dy"] = torch.randn((rows, cols), generator=g, device="cuda").to(dtype)
    elif op == "linear":
        n_in, n_out, pad = case["in"], case["out"], case["pad"]
        state["x"] = _table(g, rows, n_in, pad, dtype)
        state["w"] = _table(g, n_out, n_in, 0, dtype, n_in ** -0.5)
        state["b"] = _table(g, 1, n_out, 0, dtype, 0.3).reshape(n_out)
        state["r"] = _table(g, rows, n_out, pad, dtype) if case["residual"] else None
        state["dy"] = _table(g, rows, n_out, 0, dtype)
    else:
        cols, shots = case["cols"], case["shots"]
        t = torch.randint(0, cols, (rows, shots), generator=g, device="cuda")
        if case["kind"] == "weights":
            # outcome probabilities of random states
            re = torch.randn((rows, cols), generator=g, device="cuda")
            im = torch.randn((rows, cols), generator=g, device="cuda")
            z = re * re + im * im
            state["z"] = z / z.sum(-1, keepdim=True)
        else:
            z = 2.0 * torch.randn((rows, cols), generator=g, device="cuda")
            if case["masked"]:  # never the row's own outcome
                out = torch.rand((rows, cols), generator=g, device="cuda") < case["masked"]
                z = z.masked_fill(out.scatter(1, t, False), -math.inf)
            state["z"] = z.to(dtype)
        state["t"] = t
        state["g"] = torch.randn((rows, shots), generator=g, device="cuda") / rows
        state["gh"] = torch.randn((rows,), generator=g, device="cuda") * (0.1 / rows)
    if case["train"]:
        for k in ("x", "w", "b", "r", "z"):
            if state.get(k) is not None:
                state[k].requires_grad_(True)
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["case"]["op"]](state)


def _named(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _own_norm(s):
    from paper_2607_11985_amd import layers
    if not s["case"]["train"]:
        return _named(y=layers.layer_norm(s["x"], s["w"], s["b"], _EPS))
    y = layers.layer_norm(s["x"], s["w"], s["b"], _EPS)
    dx, dw, db = torch.autograd.grad(y, (s["x"], s["w"], s["b"]), s["dy"])
    return _named(y=y.detach(), dx=dx, dw=dw, db=db)


def _own_linear(s):
    from paper_2607_11985_amd import layers
    y = layers.linear(s["x"], s["w"], s["b"], s["case"]["act"], s["r"])
    if not s["case"]["train"]:
        return _named(y=y)
    wanted = [s["x"], s["w"], s["b"]] + ([s["r"]] if s["r"] is not None else [])
    grads = torch.autograd.grad(y, wanted, s["dy"])
    return _named(y=y.detach(), dx=grads[0], dw=grads[1], db=grads[2],
                  dr=grads[3] if len(grads) > 3 else None)


def _own_scores(s):
    from paper_2607_11985_amd import layers
    c = s["case"]
    logp, entropy, top_logp, top_index = layers.log_probs(s["z"], s["t"], top=c["top"],
                                                          kind=c["kind"])
    dz = None
    if c["train"]:
        dz, = torch.autograd.grad((logp, entropy), (s["z"],), (s["g"], s["gh"]))
    return _named(logp=logp.detach(), entropy=entropy.detach(),
                  top_logp=top_logp if c["top"] else None,
                  top_index=top_index if c["top"] else None, dz=dz)


@torch.no_grad()
def _plain_norm(s):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    centred = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + _EPS)
    h = centred * r
    y = (h * w + b).to(s["dtype"])
    if not s["case"]["train"]:
        return _named(y=y)
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    return _named(y=y, dx=dx.to(s["dtype"]), dw=(dy * h).sum(0).to(s["dtype"]),
                  db=dy.sum(0).to(s["dtype"]))


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return torch.tanh(z) if name == "tanh" else z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + \
            z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "tanh":
        t = torch.tanh(z)
        return 1 - t * t
    return torch.ones_like(z)


@torch.no_grad()
def _plain_linear(s):
    act, dtype = s["case"]["act"], s["dtype"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["b"].float()
    y = _act(act, z)
    if s["r"] is not None:
        y = y + s["r"].float()
    y = y.to(dtype)
    if not s["case"]["train"]:
        return _named(y=y)
    dz = s["dy"].float()
    if act != "none":
        dz = dz * _slope(act, z)
    return _named(y=y, dx=(dz @ w).to(dtype), dw=(dz.t() @ x).to(dtype),
                  db=dz.sum(0).to(dtype), dr=s["dy"] if s["r"] is not None else None)


def _top(z, k):
    """Indices of the k largest of each row in falling order, equal ones from the lowest index."""
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    last = torch.arange(z.shape[-1] - 1, -1, -1, device=z.device)
    return torch.topk(order * (1 << 32) + last, k, dim=-1).indices


@torch.no_grad()
def _plain_scores(s):
    c, t = s["case"], s["t"]
    z = s["z"].float()
    if c["kind"] == "weights":
        total = z.sum(-1, keepdim=True)
        p = z / total
        log_p = torch.log(p)
    else:
        m = z.amax(-1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(-1, keepdim=True)
        log_p = z - (m + torch.log(total))
        p = e / total
    product = torch.where(p > 0, p * log_p, 0.0)
    entropy = -product.sum(-1)
    out = _named(logp=log_p.gather(-1, t), entropy=entropy)
    if c["top"]:
        out["top_index"] = _top(z, c["top"])
        out["top_logp"] = log_p.gather(-1, out["top_index"])
    if c["train"]:
        dz = -p * s["g"].sum(-1, keepdim=True)
        dz -= s["gh"].unsqueeze(-1) * (product + p * entropy.unsqueeze(-1))
        dz.scatter_add_(-1, t, s["g"])
        out["dz"] = dz.to(s["dtype"])
    return {k: out[k] for k in ("logp", "entropy", "top_logp", "top_index", "dz") if k in out}


_RUN_OWN = {"layer_norm": _own_norm, "linear": _own_linear, "log_probs": _own_scores}
_RUN_PLAIN = {"layer_norm": _plain_norm, "linear": _plain_linear, "log_probs": _plain_scores}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    rows, train = case["rows"], case["train"]
    if case["op"] == "layer_norm":
        cols = case["cols"]
        # x and y; in training dy and dx; the vectors
        return {"bytes": size * (rows * cols * (4 if train else 2) + cols * (4 if train else 2)),
                "flops": rows * cols * (20 if train else 8)}
    if case["op"] == "linear":
        k, n = case["in"], case["out"]
        r = rows * n if case["residual"] else 0
        elements = rows * k + n * k + n + rows * n + r
        if train:
            elements = 2 * elements + rows * n - r  # dr is dy
        return {"bytes": size * elements, "flops": rows * k * n * (6 if train else 2)}
    cols, shots, top = case["cols"], case["shots"], case["top"]
    bytes_ = size * rows * cols * (2 if train else 1)
    bytes_ += rows * ((8 + 4) * shots + 4 + (8 + 4) * top)
    if train:
        bytes_ += rows * (4 * shots + 4)
    return {"bytes": bytes_, "flops": rows * cols * (10 if train else 5)}


# ------------------------------------------------------------- 64-bit results

@torch.no_grad()
def exact(case, seed):
    """From the definitions in 64 bits: dense products, sums over rows, sorted scores."""
    s = prepare(case, seed)
    d = {k: v.detach().to(torch.float64) for k, v in s.items()
         if isinstance(v, torch.Tensor) and k != "t"}
    if case["op"] == "layer_norm":
        out = _exact_norm(case, d)
    elif case["op"] == "linear":
        out = _exact_linear(case, d)
    else:
        out = _exact_scores(case, d, s["t"])
    return out


def _exact_norm(case, d):
    x, w, n = d["x"], d["w"], case["cols"]
    mean = x.sum(1) / n
    variance = (x * x).sum(1) / n - mean * mean
    if n == 1:
        variance = torch.zeros_like(mean)
    sd = (variance.clamp(min=0) + _EPS).sqrt()
    h = (x - mean[:, None]) / sd[:, None]
    out = {"y": torch.addcmul(d["b"].expand_as(h), h, w)}
    if case["train"]:
        dy = d["dy"]
        # the Jacobian of the normalised row, (I - 1 1'/n - h h'/n) / sd, applied to dy w
        g = dy * w
        a = (g * h).sum(1) / n
        c = g.sum(1) / n
        out["dx"] = (g - c[:, None] - h * a[:, None]) / sd[:, None]
        out["dw"] = torch.sum(dy * h, 0)
        out["db"] = torch.sum(dy, 0)
    return out


def _exact_linear(case, d):
    act = case["act"]
    z = torch.addmm(d["b"].unsqueeze(0), d["x"], d["w"].t())
    normal = torch.special.ndtr
    if act == "relu":
        y, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
    elif act == "gelu":
        y = z * normal(z)
        slope = normal(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    elif act == "silu":
        y = z * torch.sigmoid(z)
        slope = torch.sigmoid(z) + y * torch.sigmoid(-z)
    elif act == "tanh":
        y = torch.tanh(z)
        slope = 1 / torch.cosh(z) ** 2
    else:
        y, slope = z, torch.ones_like(z)
    if "r" in d:
        y = d["r"] + y
    out = {"y": y}
    if case["train"]:
        dz = d["dy"] * slope
        out["dx"] = torch.mm(dz, d["w"])
        out["dw"] = torch.mm(d["x"].t().contiguous(), dz).t()
        out["db"] = torch.sum(dz, 0)
        if "r" in d:
            out["dr"] = d["dy"]
    return out


def _exact_scores(case, d, t):
    z = d["z"]
    if case["kind"] == "weights":
        p = z / torch.sum(z, 1, keepdim=True)
        log_p = torch.log(p)
    else:
        log_p = torch.log_softmax(z, 1)
        p = torch.softmax(z, 1)
    entropy = -torch.special.xlogy(p, p).sum(1)
    out = {"logp": torch.gather(log_p, 1, t), "entropy": entropy}
    if case["top"]:
        out["top_logp"] = torch.sort(log_p, dim=1, descending=True)[0][:, :case["top"]]
        out["top_index"] = None
    if case["train"]:
        # d logp_t / dz = e_t - p;  d H / dz = -p (log p + H)
        picked = torch.zeros_like(z).scatter_add_(1, t, d["g"])
        dh = torch.special.xlogy(p, p) + p * entropy[:, None]
        out["dz"] = picked - p * d["g"].sum(1, keepdim=True) - dh * d["gh"][:, None]
    return out
