"""Serving a hybrid model: its linear layers in 8-bit integers, and its answers from drafted
outcomes that are verified against the model's own probabilities.

`linear_quantized`: rows are quantised within the call, each by its own largest magnitude, and
multiplied with weights that were quantised once, each output channel by its own; bias, activation
and residual follow in the same call.  `verify_drafts`: outcomes that a cheaper model drafted are
accepted one after the other with given uniform numbers, and the first that is not is replaced by
one drawn from what the draft's probabilities leave of the target's.  In the plain form both are
elementary torch operations; with `own` set the calls are those of paper_2607_11985_amd.layers.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# bounds of the drawn cases: products, weights and scores of the largest listed ones
_MOST_PRODUCTS = 512 * 4096 * 65536
_MOST_WEIGHTS = 4096 * 65536
_MOST_SCORES = 64 * 15 * 128000


def _linear(rows, n_in, n_out, dtype, act="none", residual=False, pad=0):
    return {"op": "linear_quantized", "rows": rows, "in": n_in, "out": n_out, "dtype": dtype,
            "act": act, "residual": residual, "pad": pad}


def _verify(sequences, drafts, cols, dtype, kind="logits", temperature=1.0, ragged=False,
            masked=0.0):
    return {"op": "verify_drafts", "sequences": sequences, "drafts": drafts, "cols": cols,
            "dtype": dtype, "kind": kind, "temperature": temperature, "ragged": ragged,
            "masked": masked}


def listed():
    return [
        # 16 expectations to 10 logits, the smallest read-out: latency
        dict(_linear(64, 16, 10, "f32"), name="linear_f32_64x16x10"),
        # one sample's wide features through a square layer with its residual
        dict(_linear(1, 4096, 4096, "bf16", "gelu", True), name="linear_bf16_1x4096x4096"),
        # the logits of 2^16 outcomes at the five positions of one sequence's four drafts: the
        # weights are all there is to read
        dict(_linear(5, 4096, 65536, "bf16"), name="linear_bf16_5x4096x65536"),
        # 2^14 outcome probabilities of a batch read out into classes: a long sum, few outputs
        dict(_linear(301, 16384, 101, "f16"), name="linear_f16_301x16384x101"),
        # odd sizes throughout, features out of a wider table
        dict(_linear(1000, 1001, 1003, "bf16", "silu", pad=3), name="linear_bf16_1000x1001x1003"),
        # features to the 384 per-sample angles of a 16-qubit, 8-layer circuit
        dict(_linear(1024, 768, 384, "f32", "tanh"), name="linear_f32_1024x768x384"),
        # a wide layer over a large batch
        dict(_linear(8192, 4096, 4096, "bf16", "gelu", True), name="linear_bf16_8192x4096x4096"),
        # the logits of 2^16 outcomes for 64 sequences of seven drafts each
        dict(_linear(512, 4096, 65536, "bf16"), name="linear_bf16_512x4096x65536"),
        # three drafted outcomes of one 10-qubit state: latency
        dict(_verify(1, 3, 1024, "f32", "weights"), name="verify_weights_f32_1x3x1024"),
        # outcomes of 16-qubit states drafted from shallower circuits
        dict(_verify(32, 4, 65536, "f32", "weights"), name="verify_weights_f32_32x4x65536"),
        # sequences with fewer drafts than the widest, an odd number of outcomes, some ruled out
        dict(_verify(37, 5, 50001, "f16", temperature=0.5, ragged=True, masked=0.1),
             name="verify_f16_37x5x50001"),
        # a full batch over many outcomes
        dict(_verify(64, 7, 128000, "bf16"), name="verify_bf16_64x7x128000"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        dtype = rng.choice(["f32", "f16", "bf16"])
        if rng.random() < 0.6:
            case = _linear(log_int(1, 8192), log_int(1, 16384), log_int(1, 65536), dtype,
                           rng.choice(["none", "relu", "gelu", "silu", "tanh"]),
                           rng.random() < 0.5, rng.choice([0, 0, 1, 8]))
            weights = case["in"] * case["out"]
            if weights <= _MOST_WEIGHTS and case["rows"] * weights <= _MOST_PRODUCTS:
                return case
        else:
            kind = rng.choice(["logits", "logits", "weights"])
            cols = 1 << rng.randint(4, 20) if kind == "weights" else log_int(2, 1 << 18)
            case = _verify(log_int(1, 256), rng.randint(0, 8), cols,
                           "f32" if kind == "weights" else dtype, kind,
                           rng.choice([1.0, 0.5, 0.8]) if kind == "logits" else 1.0,
                           rng.random() < 0.3,
                           rng.choice([0.0, 0.3]) if kind == "logits" else 0.0)
            if case["sequences"] * (2 * case["drafts"] + 1) * cols <= _MOST_SCORES:
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
    g, dtype = _generator(seed), _TYPES[case["dtype"]]
    state = {"case": case, "dtype": dtype}
    return (_prepare_linear if case["op"] == "linear_quantized" else _prepare_verify)(
        case, g, dtype, state)


def _prepare_linear(case, g, dtype, state):
    rows, n_in, n_out, pad = case["rows"], case["in"], case["out"], case["pad"]
    # rows of unlike level
    x = torch.randn((rows, n_in + pad), generator=g, device="cuda")
    x *= torch.rand((rows, 1), generator=g, device="cuda") * 2 + 0.5
    state["x"] = x.to(dtype)[:, :n_in]
    w = torch.randn((n_out, n_in), generator=g, device="cuda") * n_in ** -0.5
    w *= torch.rand((n_out, 1), generator=g, device="cuda") + 0.5
    if own:
        from paper_2607_11985_amd import layers
        state["w"] = layers.quantize(w)
    else:
        state["w"] = _quantized(w)
    state["b"] = _table(g, 1, n_out, 0, dtype, 0.3).reshape(n_out)
    state["r"] = _table(g, rows, n_out, 0, dtype) if case["residual"] else None
    return state


def _prepare_verify(case, g, dtype, state):
    n, k, cols = case["sequences"], case["drafts"], case["cols"]
    target = 2.0 * torch.randn((n, k + 1, cols), generator=g, device="cuda")
    # the draft is near the target, but not the same
    draft = target[:, :k] + 0.7 * torch.randn((n, k, cols), generator=g, device="cuda")
    if case["masked"]:
        out = torch.rand((1, 1, cols), generator=g, device="cuda") < case["masked"]
        out[..., 0] = False
        target, draft = target.masked_fill(out, -math.inf), draft.masked_fill(out, -math.inf)
    if case["kind"] == "weights":
        # outcome probabilities of states
        target = torch.softmax(target, -1)
        draft = torch.softmax(draft, -1)
        noisy = torch.log(draft)
    else:
        target, draft = target.to(dtype), draft.to(dtype)
        noisy = draft.float() * (1.0 / case["temperature"])
    # outcomes drawn from the draft
    e = torch.rand((n, k, cols), generator=g, device="cuda").clamp_(min=1e-30)
    noisy = noisy - torch.log(-torch.log(e))
    d = noisy.argmax(-1) if k else torch.empty((n, 0), dtype=torch.int64, device="cuda")
    if case["ragged"] and k:
        some = torch.randint(0, k + 1, (n, 1), generator=g, device="cuda")
        d = torch.where(torch.arange(k, device="cuda") < some, d, -1)
    state["target"], state["draft"], state["drafted"] = target, draft, d
    state["u"] = torch.rand((n, k + 1), generator=g, device="cuda", dtype=torch.float64)
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["case"]["op"]](state)


def _own_linear(s):
    from paper_2607_11985_amd import layers
    return {"y": layers.linear_quantized(s["x"], s["w"], s["b"], s["case"]["act"], s["r"])}


def _own_verify(s):
    from paper_2607_11985_amd import layers
    c = s["case"]
    outcomes, accepted = layers.verify_drafts(s["target"], s["draft"], s["drafted"], s["u"],
                                              kind=c["kind"], temperature=c["temperature"])
    return {"outcomes": outcomes, "accepted": accepted}


def _quantized(x):
    """Integers in [-127, 127] and the step of each row.  The quotients are 64-bit: beside the
    border between two integers a 32-bit one falls to the wrong side."""
    most = x.abs().amax(-1, keepdim=True)
    q = torch.round(127.0 * x.double() / torch.where(most > 0, most, 1.0).double())
    return q.to(torch.int8), (most.float() / 127.0).squeeze(-1)


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return torch.tanh(z) if name == "tanh" else z


@torch.no_grad()
def _plain_linear(s):
    xq, xs = _quantized(s["x"])
    wq, ws = s["w"]
    z = (xq.float() @ wq.float().t()) * xs[:, None] * ws + s["b"].float()
    y = _act(s["case"]["act"], z)
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(s["dtype"])}


def _probabilities(scores, kind, temperature):
    w = scores.double()
    if kind == "logits":
        w = torch.exp((w - w.amax(-1, keepdim=True)) / temperature)
    return w / w.sum(-1, keepdim=True)


@torch.no_grad()
def _plain_verify(s):
    """64-bit throughout: a cumulative sum that is a little off turns some draws into their
    neighbours."""
    c, d, u = s["case"], s["drafted"], s["u"]
    n, k = d.shape
    p = _probabilities(s["target"], c["kind"], c["temperature"])
    q = _probabilities(s["draft"], c["kind"], c["temperature"])
    there = (d >= 0) & (d < c["cols"])
    at = torch.where(there, d, 0).unsqueeze(-1)
    ok = there & (u[:, :k] * q.gather(-1, at).squeeze(-1) < p[:, :k].gather(-1, at).squeeze(-1))
    accepted = ok.long().cumprod(-1).sum(-1)
    every = torch.arange(n, device=d.device)
    left = p[every, accepted]
    if k:
        last = accepted.clamp(max=k - 1)
        rejected = (accepted < k) & there[every, last]
        rest = (left - q[every, last]).clamp(min=0)
        left = torch.where(rejected[:, None] & (rest.sum(-1, keepdim=True) > 0), rest, left)
    sums = left.cumsum(-1)
    drawn = (sums > u[:, k:] * sums[:, -1:]).long().argmax(-1)
    place = torch.arange(k + 1, device=d.device)
    drafts = torch.cat([d, d.new_full((n, 1), -1)], 1)
    outcomes = torch.where(place < accepted[:, None], drafts,
                           torch.where(place == accepted[:, None], drawn[:, None], -1))
    return {"outcomes": outcomes, "accepted": accepted}


_RUN_OWN = {"linear_quantized": _own_linear, "verify_drafts": _own_verify}
_RUN_PLAIN = {"linear_quantized": _plain_linear, "verify_drafts": _plain_verify}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "linear_quantized":
        m, k, n = case["rows"], case["in"], case["out"]
        outputs = m * n * (2 if case["residual"] else 1)
        # rows, bias, residual and result; weights and their steps
        return {"bytes": size * (m * k + n + outputs) + n * k + 4 * n, "flops": 2 * m * n * k}
    n, k, cols = case["sequences"], case["drafts"], case["cols"]
    scores = n * (2 * k + 1) * cols
    # drafts and uniform numbers; outcomes and how many drafts were accepted
    return {"bytes": size * scores + 8 * n * (k + k + 1) + 8 * n * (k + 2), "flops": 5 * scores}


# ------------------------------------------------------------- 64-bit results

@torch.no_grad()
def exact(case, seed):
    """The linear layers from their definition in 64 bits, on the numbers that the integers stand
    for.  Outcomes are whole numbers."""
    if case["op"] == "verify_drafts":
        return None
    s = prepare(case, seed)
    x, w = s["x"].to(torch.float64), s["w"]
    step = torch.linalg.vector_norm(x, math.inf, dim=1, keepdim=True) / 127
    integers = torch.div(x, torch.where(step == 0, 1.0, step))
    # a quotient by the rounded step may miss a tie: ties are those of the exact products
    n = integers.round()
    for _ in range(2):
        far = 2 * (127 * x - n * (127 * step))
        size = 127 * step
        n = n + ((far > size) | ((far == size) & (n % 2 != 0))).double()
        n = n - ((far < -size) | ((far == -size) & (n % 2 != 0))).double()
    z = torch.mm(n * step, (w[0].double() * w[1].double()[:, None]).t())
    z = z + s["b"].double()
    act = case["act"]
    if act == "relu":
        z = torch.where(z > 0, z, 0.0)
    elif act == "gelu":
        z = z * torch.special.ndtr(z)
    elif act == "silu":
        z = z * torch.sigmoid(z)
    elif act == "tanh":
        z = torch.tanh(z)
    return {"y": z if s["r"] is None else s["r"].double() + z}
