"""Layers around a circuit, computed in libvqc.so and differentiable through torch.autograd.

    h = layer_norm(features, w, b)                       # features before the encoding
    angles = linear(h, W, bias, activation="tanh")       # features -> angles
    E = VQCFunction.apply(circ, params, angles)
    logits = linear(E, V, c)                             # read-out
    s = log_probs(logits, labels, top=3)                 # s.logp, s.entropy, s.top_logp, ...
    (-s.logp.mean()).backward()

Tensors are cuda tensors of one type (float32, float16 or bfloat16); statistics and sums are
float32.  Leading dimensions are rows.  Rows may be any distance apart; a row's elements must be
adjacent.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

from . import _lib
from .api import _stream

_DTYPES = {torch.float32: _lib.DTYPE["float32"], torch.float16: _lib.DTYPE["float16"],
           torch.bfloat16: _lib.DTYPE["bfloat16"]}


class LogProbs(NamedTuple):
    """What log_probs returns."""
    logp: torch.Tensor        # log probabilities of the targets, float32, their shape
    entropy: torch.Tensor     # [rows...] float32
    top_logp: torch.Tensor    # [rows..., top] float32, falling
    top_index: torch.Tensor   # [rows..., top] int64


def _type_of(x, name):
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a cuda tensor")
    return code


def _like(x, like, name):
    if x.dtype is not like.dtype or x.device != like.device:
        raise ValueError(f"{name} must be {like.dtype} on {like.device}, got {x.dtype} on "
                         f"{x.device}")


def _matrix(x, width, name):
    """x as [rows, width], each row's elements adjacent (a copy only where leading dimensions do
    not merge)."""
    if x.dim() < 1 or x.shape[-1] != width:
        raise ValueError(f"{name} must have rows of {width}, got {tuple(x.shape)}")
    if width > 1 and x.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {name} must be adjacent, got strides "
                         f"{x.stride()}")
    if x.dim() == 2:
        return x
    return x.reshape(-1, width) if width else x.reshape(math.prod(x.shape[:-1]), 0)


def _vector(x, width, like, name):
    if x.dtype is not like.dtype or x.device != like.device or x.shape != (width,) or \
            not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {like.dtype} tensor of {width} elements "
                         f"on {like.device}")
    return x


def _cotangent(g, rows, width, dtype):
    """A cotangent as adjacent-element rows (autograd may hand over expanded tensors)."""
    if g.dim() != 2:
        g = g.reshape(rows, width)
    if g.dtype is not dtype:
        g = g.to(dtype)
    return g if width <= 1 or g.stride(1) == 1 else g.contiguous()


def _run(device, fn, args):
    """fn(*args, stream) on the current stream of `device`, with that device current."""
    if device.index == torch.cuda.current_device():
        rc = fn(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(device))
    if rc:
        _lib._check(rc)


def _once(backward):
    """A backward that is not differentiable itself: with create_graph autograd is told so
    (otherwise grad mode is off here already, and the check costs nothing)."""
    checked = torch.autograd.function.once_differentiable(backward)

    def apply(ctx, *grads):
        return checked(ctx, *grads) if torch.is_grad_enabled() else backward(ctx, *grads)
    return staticmethod(apply)


# ------------------------------------------------------------------ layer norm

def _layer_norm_forward(x, weight, bias, eps, keep):
    """y, and with keep (rows, cols, row stride, mean and rstd)."""
    code = _type_of(x, "x")
    if not x.dim() or x.shape[-1] < 1:
        raise ValueError(f"x must have rows of at least one element, got {tuple(x.shape)}")
    cols = x.shape[-1]
    xm = _matrix(x, cols, "x")
    rows, ld = xm.shape[0], xm.stride(0)
    wp = _vector(weight, cols, x, "weight").data_ptr() if weight is not None else None
    bp = _vector(bias, cols, x, "bias").data_ptr() if bias is not None else None
    device = x.device
    y = torch.empty(x.shape, dtype=x.dtype, device=device)
    stats = mean = rstd = None
    if keep:
        stats = torch.empty((2, rows), dtype=torch.float32, device=device)
        mean = stats.data_ptr()
        rstd = mean + 4 * rows
    _run(device, _lib.load().vqc_layer_norm,
         (code, rows, cols, xm.data_ptr(), ld, wp, bp, eps, y.data_ptr(), cols, mean, rstd))
    return y, stats


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, ctx.stats = _layer_norm_forward(x, weight, bias, eps, True)
        ctx.save_for_backward(x, weight)
        return y

    @_once
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        stats = ctx.stats
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        cols, dtype, device = x.shape[-1], x.dtype, x.device
        xm = x if x.dim() == 2 else _matrix(x, cols, "x")
        rows = xm.shape[0]
        dym = _cotangent(dy, rows, cols, dtype)
        dx = dw = db = ws = None
        dxp = dwp = dbp = wsp = None
        if need_x:
            dx = torch.empty(x.shape, dtype=dtype, device=device)
            dxp = dx.data_ptr()
        if need_w:
            dw = torch.empty(cols, dtype=dtype, device=device)
            dwp = dw.data_ptr()
        if need_b:
            db = torch.empty(cols, dtype=dtype, device=device)
            dbp = db.data_ptr()
        lib = _lib.load()
        nb = 0
        if need_w or need_b:
            nb = lib.vqc_layer_norm_workspace_bytes(rows, cols)
            if nb:
                ws = torch.empty(nb, dtype=torch.uint8, device=device)
                wsp = ws.data_ptr()
        mean = stats.data_ptr()
        _run(device, lib.vqc_layer_norm_backward,
             (_DTYPES[dtype], rows, cols, xm.data_ptr(), xm.stride(0),
              weight.data_ptr() if weight is not None else None, mean, mean + 4 * rows,
              dym.data_ptr(), dym.stride(0), dxp, cols, dwp, dbp, wsp, nb))
        return dx, dw, db, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the last dimension."""
    if torch.is_grad_enabled() and (x.requires_grad or
                                    (weight is not None and weight.requires_grad) or
                                    (bias is not None and bias.requires_grad)):
        return LayerNormFunction.apply(x, weight, bias, float(eps))
    return _layer_norm_forward(x, weight, bias, float(eps), False)[0]


# ------------------------------------------------------------------ linear

def _linear_forward(x, weight, bias, act, residual, keep):
    """y, and with keep the activation's argument where the backward needs it."""
    code = _type_of(x, "x")
    if weight.dim() != 2:
        raise ValueError(f"weight must be [n_out, n_in], got {tuple(weight.shape)}")
    n_out, n_in = weight.shape
    xm = _matrix(x, n_in, "x")
    _like(weight, x, "weight")
    _matrix(weight, n_in, "weight")
    bp = _vector(bias, n_out, x, "bias").data_ptr() if bias is not None else None
    rows, device = xm.shape[0], x.device
    shape = (rows, n_out) if x.dim() == 2 else x.shape[:-1] + (n_out,)
    rp, ldr = None, 0
    if residual is not None:
        if residual.shape != shape:
            raise ValueError(f"residual must have shape {tuple(shape)}, got "
                             f"{tuple(residual.shape)}")
        _like(residual, x, "residual")
        rm = _matrix(residual, n_out, "residual")
        rp, ldr = rm.data_ptr(), rm.stride(0)
    y = torch.empty(shape, dtype=x.dtype, device=device)
    pre = torch.empty((rows, n_out), dtype=torch.float32, device=device) if keep and act else None
    lib = _lib.load()
    nb, wsp = lib.vqc_linear_workspace_bytes(code, rows, n_in, n_out, 0), None
    if nb:
        ws = torch.empty(nb, dtype=torch.uint8, device=device)
        wsp = ws.data_ptr()
    _run(device, lib.vqc_linear,
         (code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0), weight.data_ptr(),
          weight.stride(0), bp, act, rp, ldr, y.data_ptr(), n_out,
          pre.data_ptr() if pre is not None else None, wsp, nb))
    return y, pre


class LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, residual):
        y, ctx.pre = _linear_forward(x, weight, bias, act, residual, True)
        ctx.save_for_backward(x, weight)
        ctx.act = act
        return y

    @_once
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        pre = ctx.pre
        n_out, n_in = weight.shape
        need_x, need_w, need_b, _, need_r = ctx.needs_input_grad
        dx = dw = db = None
        if need_x or need_w or need_b:
            dtype, device = x.dtype, x.device
            code = _DTYPES[dtype]
            xm = x if x.dim() == 2 else _matrix(x, n_in, "x")
            rows = xm.shape[0]
            dym = _cotangent(dy, rows, n_out, dtype)
            dxp = dwp = dbp = wsp = None
            if need_x:
                dx = torch.empty(x.shape, dtype=dtype, device=device)
                dxp = dx.data_ptr()
            if need_w:
                dw = torch.empty((n_out, n_in), dtype=dtype, device=device)
                dwp = dw.data_ptr()
            if need_b:
                db = torch.empty(n_out, dtype=dtype, device=device)
                dbp = db.data_ptr()
            lib = _lib.load()
            nb = lib.vqc_linear_workspace_bytes(code, rows, n_in, n_out, 1)
            if nb:
                ws = torch.empty(nb, dtype=torch.uint8, device=device)
                wsp = ws.data_ptr()
            _run(device, lib.vqc_linear_backward,
                 (code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0), weight.data_ptr(),
                  weight.stride(0), ctx.act, pre.data_ptr() if pre is not None else None,
                  dym.data_ptr(), dym.stride(0), dxp, n_in, dwp, n_in, dbp, wsp, nb))
        return dx, dw, db, None, dy if need_r else None


def linear(x, weight, bias=None, activation: str = "none", residual=None):
    """activation(x weight^T + bias) + residual, activation one of none, relu, gelu, silu, tanh."""
    act = _lib.ACT.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(_lib.ACT)}, got {activation!r}")
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                    (bias is not None and bias.requires_grad) or
                                    (residual is not None and residual.requires_grad)):
        return LinearFunction.apply(x, weight, bias, act, residual)
    return _linear_forward(x, weight, bias, act, residual, False)[0]


# ------------------------------------------------------------------ scores

def _log_probs_forward(scores, targets, top, kind, inv_t, keep):
    """(logp, entropy, top_logp, top_index), the targets as read, their number per row, and
    with keep the rows' statistics."""
    code = _type_of(scores, "scores")
    if not scores.dim() or scores.shape[-1] < 1:
        raise ValueError(f"scores must have rows of at least one outcome, got "
                         f"{tuple(scores.shape)}")
    cols, lead, device = scores.shape[-1], scores.shape[:-1], scores.device
    if not 0 <= top <= min(cols, _lib.VQC_MAX_TOP):
        raise ValueError(f"top must be in [0, min({cols}, {_lib.VQC_MAX_TOP})], got {top}")
    sm = _matrix(scores, cols, "scores")
    rows = sm.shape[0]
    f32 = torch.float32
    shots, tp, lp = 0, None, None
    if targets is None:
        logp = torch.empty(lead + (0,), dtype=f32, device=device)
    else:
        if targets.dtype is not torch.int64 or targets.device != device:
            raise ValueError(f"targets must be int64 on {device}, got {targets.dtype} on "
                             f"{targets.device}")
        if targets.shape == lead:
            shots = 1
        elif targets.dim() == len(lead) + 1 and targets.shape[:-1] == lead:
            shots = targets.shape[-1]
        else:
            raise ValueError(f"targets must have shape {tuple(lead)} or {tuple(lead)} + (n,), "
                             f"got {tuple(targets.shape)}")
        targets = targets.contiguous()
        logp = torch.empty(targets.shape, dtype=f32, device=device)
        if shots:
            tp, lp = targets.data_ptr(), logp.data_ptr()
    entropy = torch.empty(lead, dtype=f32, device=device)
    top_logp = torch.empty(lead + (top,), dtype=f32, device=device)
    top_index = torch.empty(lead + (top,), dtype=torch.int64, device=device)
    stats = torch.empty((rows, 2), dtype=f32, device=device) if keep else None
    lib = _lib.load()
    nb, wsp = lib.vqc_log_probs_workspace_bytes(rows, cols, top), None
    if nb:
        ws = torch.empty(nb, dtype=torch.uint8, device=device)
        wsp = ws.data_ptr()
    _run(device, lib.vqc_log_probs,
         (kind, code, rows, cols, sm.data_ptr(), sm.stride(0), inv_t, tp, shots, lp,
          entropy.data_ptr(), top, top_logp.data_ptr() if top else None,
          top_index.data_ptr() if top else None, stats.data_ptr() if keep else None, wsp, nb))
    return (logp, entropy, top_logp, top_index), targets, shots, stats


class LogProbsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, targets, top, inv_t):
        out, targets, shots, stats = _log_probs_forward(scores, targets, top,
                                                        _lib.SCORES["logits"], inv_t, True)
        ctx.save_for_backward(scores, targets, out[1])
        ctx.kept = stats, shots, inv_t
        ctx.mark_non_differentiable(out[2], out[3])
        ctx.set_materialize_grads(False)
        return out

    @_once
    def backward(ctx, dlogp, dentropy, _top_logp, _top_index):
        if dlogp is None and dentropy is None:
            return None, None, None, None
        scores, targets, entropy = ctx.saved_tensors
        stats, shots, inv_t = ctx.kept
        cols, device = scores.shape[-1], scores.device
        sm = scores if scores.dim() == 2 else _matrix(scores, cols, "scores")
        dz = torch.empty(scores.shape, dtype=scores.dtype, device=device)
        g = dlogp.contiguous() if dlogp is not None and shots else None
        gh = dentropy.contiguous() if dentropy is not None else None
        _run(device, _lib.load().vqc_log_probs_backward,
             (_DTYPES[scores.dtype], sm.shape[0], cols, sm.data_ptr(), sm.stride(0), inv_t,
              targets.data_ptr() if g is not None else None, shots, stats.data_ptr(),
              entropy.data_ptr(), g.data_ptr() if g is not None else None,
              gh.data_ptr() if gh is not None else None, dz.data_ptr(), cols))
        return dz, None, None, None


def log_probs(scores, targets: Optional[torch.Tensor] = None, top: int = 0,
              kind: str = "logits", temperature: float = 1.0) -> LogProbs:
    """Log probabilities of the target outcomes, entropy and the `top` most probable outcomes.

    scores [..., outcomes]: logits, or with kind="weights" unnormalised probabilities such as
    those of Circuit.forward_ex (no gradient).  targets [...] or [..., n] int64, -1 for none.
    logp and entropy are differentiable with respect to logits."""
    code = _lib.SCORES.get(kind)
    if code is None:
        raise ValueError(f"kind must be one of {sorted(_lib.SCORES)}, got {kind!r}")
    if not (temperature > 0 and math.isfinite(temperature)):
        raise ValueError(f"temperature must be finite and positive, got {temperature}")
    if code and temperature != 1.0:
        raise ValueError("weights have no temperature")
    if scores.requires_grad and torch.is_grad_enabled():
        if code:
            raise ValueError("weights have no gradient here: detach them, or give logits")
        return LogProbs(*LogProbsFunction.apply(scores, targets, int(top), 1.0 / temperature))
    return LogProbs(*_log_probs_forward(scores, targets, int(top), code, 1.0 / temperature,
                                        False)[0])
