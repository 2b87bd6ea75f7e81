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
from .api import _ptr, _stream

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


def _as_matrix(x, width, like, name):
    """x as rows of `width` adjacent elements, [rows, width] (a copy only where leading
    dimensions do not merge)."""
    if x.dtype != like.dtype or x.device != like.device:
        raise ValueError(f"{name} must be {like.dtype} on {like.device}, got {x.dtype} on "
                         f"{x.device}")
    if x.dim() < 1 or x.shape[-1] != width:
        raise ValueError(f"{name} must have rows of {width}, got {tuple(x.shape)}")
    if width > 1 and x.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {name} must be adjacent, got strides "
                         f"{x.stride()}")
    return x if x.dim() == 2 else x.reshape(-1, width) if width else \
        x.reshape(math.prod(x.shape[:-1]), 0)


def _as_vector(x, width, like, name):
    if x is None:
        return None
    if x.dtype != like.dtype or x.device != like.device or tuple(x.shape) != (width,) or \
            not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {like.dtype} tensor of {width} elements "
                         f"on {like.device}")
    return x


def _rows_of(g, like_shape, dtype):
    """A cotangent as adjacent-element rows (autograd may hand over expanded tensors)."""
    g = g.reshape(like_shape)
    if g.dtype != dtype:
        g = g.to(dtype)
    return g if g.shape[-1] <= 1 or g.stride(-1) == 1 else g.contiguous()


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _on(device):
    """The device of the tensors as the current one."""
    return torch.cuda.device(device)


def _current(device):
    return device.index is None or device.index == torch.cuda.current_device()


def _call(device, fn, *args):
    """fn(*args, stream) with `device` current."""
    if _current(device):
        return fn(*args, _stream(device))
    with _on(device):
        return fn(*args, _stream(device))


def _wants_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ------------------------------------------------------------------ layer norm

def _layer_norm_forward(x, weight, bias, eps, keep):
    code = _type_of(x, "x")
    cols = x.shape[-1] if x.dim() else 0
    if cols < 1:
        raise ValueError(f"x must have rows of at least one element, got {tuple(x.shape)}")
    xm = _as_matrix(x, cols, x, "x")
    weight = _as_vector(weight, cols, x, "weight")
    bias = _as_vector(bias, cols, x, "bias")
    rows = xm.shape[0]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = rstd = None
    if keep:
        mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device)
    _call(x.device, _lib.vqc_layer_norm, code, rows, cols, xm.data_ptr(), xm.stride(0),
          _ptr(weight), _ptr(bias), eps, y.data_ptr(), cols, _ptr(mean), _ptr(rstd))
    return y, xm, mean, rstd


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, xm, mean, rstd = _layer_norm_forward(x, weight, bias, eps, True)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        cols = x.shape[-1]
        xm = _as_matrix(x, cols, x, "x")
        rows = xm.shape[0]
        dym = _rows_of(dy, (rows, cols), x.dtype)
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        new = dict(dtype=x.dtype, device=x.device)
        dx = torch.empty(x.shape, **new) if need_x else None
        dw = torch.empty(cols, **new) if need_w and weight is not None else None
        db = torch.empty(cols, **new) if need_b and ctx.has_bias else None
        nb = _lib.vqc_layer_norm_workspace_bytes(rows, cols) if dw is not None or db is not None \
            else 0
        ws = _workspace(nb, x.device)
        _call(x.device, _lib.vqc_layer_norm_backward, _DTYPES[x.dtype], rows, cols, xm.data_ptr(),
              xm.stride(0), _ptr(weight), mean.data_ptr(), rstd.data_ptr(), dym.data_ptr(),
              dym.stride(0), _ptr(dx), cols, _ptr(dw), _ptr(db), _ptr(ws), nb)
        return dx, dw, db, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the last dimension."""
    if _wants_grad(x, weight, bias):
        return LayerNormFunction.apply(x, weight, bias, float(eps))
    return _layer_norm_forward(x, weight, bias, float(eps), False)[0]


# ------------------------------------------------------------------ linear

def _linear_forward(x, weight, bias, act, residual, keep):
    code = _type_of(x, "x")
    if weight.dim() != 2:
        raise ValueError(f"weight must be [n_out, n_in], got {tuple(weight.shape)}")
    n_out, n_in = weight.shape
    xm = _as_matrix(x, n_in, x, "x")
    wm = _as_matrix(weight, n_in, x, "weight")
    bias = _as_vector(bias, n_out, x, "bias")
    rows = xm.shape[0]
    shape = x.shape[:-1] + (n_out,)
    rm = None
    if residual is not None:
        if residual.shape != shape:
            raise ValueError(f"residual must have shape {tuple(shape)}, got "
                             f"{tuple(residual.shape)}")
        rm = _as_matrix(residual, n_out, x, "residual")
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    pre = torch.empty((rows, n_out), dtype=torch.float32, device=x.device) if keep and act \
        else None
    nb = _lib.vqc_linear_workspace_bytes(code, rows, n_in, n_out, 0)
    ws = _workspace(nb, x.device)
    _call(x.device, _lib.vqc_linear, code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0),
          wm.data_ptr(), wm.stride(0), _ptr(bias), act, _ptr(rm),
          rm.stride(0) if rm is not None else 0, y.data_ptr(), n_out, _ptr(pre), _ptr(ws), nb)
    return y, pre


class LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, residual):
        y, pre = _linear_forward(x, weight, bias, act, residual, True)
        ctx.save_for_backward(x, weight, pre)
        ctx.act = act
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, pre = ctx.saved_tensors
        n_out, n_in = weight.shape
        xm = _as_matrix(x, n_in, x, "x")
        rows = xm.shape[0]
        need_x, need_w, need_b, _, need_r = ctx.needs_input_grad
        dx = dw = db = None
        if need_x or need_w or need_b:
            code = _DTYPES[x.dtype]
            new = dict(dtype=x.dtype, device=x.device)
            dym = _rows_of(dy, (rows, n_out), x.dtype)
            dx = torch.empty(x.shape, **new) if need_x else None
            dw = torch.empty((n_out, n_in), **new) if need_w else None
            db = torch.empty(n_out, **new) if need_b else None
            nb = _lib.vqc_linear_workspace_bytes(code, rows, n_in, n_out, 1)
            ws = _workspace(nb, x.device)
            _call(x.device, _lib.vqc_linear_backward, code, rows, n_in, n_out, xm.data_ptr(),
                  xm.stride(0), weight.data_ptr(), weight.stride(0), ctx.act, _ptr(pre),
                  dym.data_ptr(), dym.stride(0), _ptr(dx), n_in, _ptr(dw), n_in, _ptr(db),
                  _ptr(ws), nb)
        return dx, dw, db, None, dy if need_r else None


def linear(x, weight, bias=None, activation: str = "none", residual=None):
    """activation(x weight^T + bias) + residual, activation one of none, relu, gelu, silu, tanh."""
    act = _lib.ACT.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(_lib.ACT)}, got {activation!r}")
    if _wants_grad(x, weight, bias, residual):
        return LinearFunction.apply(x, weight, bias, act, residual)
    return _linear_forward(x, weight, bias, act, residual, False)[0]


# ------------------------------------------------------------------ scores

def _log_probs_forward(scores, targets, top, kind, inv_t, keep):
    code = _type_of(scores, "scores")
    cols = scores.shape[-1] if scores.dim() else 0
    if cols < 1:
        raise ValueError(f"scores must have rows of at least one outcome, got "
                         f"{tuple(scores.shape)}")
    if not 0 <= top <= min(cols, _lib.VQC_MAX_TOP):
        raise ValueError(f"top must be in [0, min({cols}, {_lib.VQC_MAX_TOP})], got {top}")
    lead = scores.shape[:-1]
    sm = _as_matrix(scores, cols, scores, "scores")
    rows = sm.shape[0]
    shots = 0
    if targets is not None:
        if targets.dtype != torch.int64 or targets.device != scores.device:
            raise ValueError(f"targets must be int64 on {scores.device}, got {targets.dtype} on "
                             f"{targets.device}")
        if targets.shape == lead:
            shots = 1
        elif targets.dim() == len(lead) + 1 and targets.shape[:-1] == lead:
            shots = targets.shape[-1]
        else:
            raise ValueError(f"targets must have shape {tuple(lead)} or {tuple(lead)} + (n,), "
                             f"got {tuple(targets.shape)}")
        targets = targets.contiguous()
    new = dict(dtype=torch.float32, device=scores.device)
    logp = torch.empty(lead if targets is None else targets.shape, **new) if shots else \
        torch.empty(lead + (0,), **new)
    entropy = torch.empty(lead, **new)
    top_logp = torch.empty(lead + (top,), **new)
    top_index = torch.empty(lead + (top,), dtype=torch.int64, device=scores.device)
    stats = torch.empty((rows, 2), **new) if keep else None
    nb = _lib.vqc_log_probs_workspace_bytes(rows, cols, top)
    ws = _workspace(nb, scores.device)
    _call(scores.device, _lib.vqc_log_probs, kind, code, rows, cols, sm.data_ptr(), sm.stride(0),
          inv_t, _ptr(targets) if shots else None, shots, logp.data_ptr() if shots else None,
          entropy.data_ptr(), top, top_logp.data_ptr() if top else None,
          top_index.data_ptr() if top else None, _ptr(stats), _ptr(ws), nb)
    return LogProbs(logp, entropy, top_logp, top_index), targets, shots, stats


class LogProbsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, targets, top, inv_t):
        out, targets, shots, stats = _log_probs_forward(scores, targets, top,
                                                        _lib.SCORES["logits"], inv_t, True)
        ctx.save_for_backward(scores, targets, stats, out.entropy)
        ctx.inv_t = inv_t
        ctx.shots = shots
        ctx.mark_non_differentiable(out.top_logp, out.top_index)
        ctx.set_materialize_grads(False)
        return tuple(out)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy, _top_logp, _top_index):
        if dlogp is None and dentropy is None:
            return None, None, None, None
        scores, targets, stats, entropy = ctx.saved_tensors
        cols = scores.shape[-1]
        sm = _as_matrix(scores, cols, scores, "scores")
        rows = sm.shape[0]
        dz = torch.empty(scores.shape, dtype=scores.dtype, device=scores.device)
        g = dlogp.contiguous() if dlogp is not None and ctx.shots else None
        gh = dentropy.contiguous() if dentropy is not None else None
        _call(scores.device, _lib.vqc_log_probs_backward, _DTYPES[scores.dtype], rows, cols,
              sm.data_ptr(), sm.stride(0), ctx.inv_t, _ptr(targets), ctx.shots, stats.data_ptr(),
              entropy.data_ptr(), _ptr(g), _ptr(gh), dz.data_ptr(), cols)
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
    if _wants_grad(scores):
        if code:
            raise ValueError("weights have no gradient here: detach them, or give logits")
        return LogProbs(*LogProbsFunction.apply(scores, targets, int(top), 1.0 / temperature))
    return _log_probs_forward(scores, targets, int(top), code, 1.0 / temperature, False)[0]
