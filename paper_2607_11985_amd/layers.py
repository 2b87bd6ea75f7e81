"""Layers around a circuit, computed in libvqc.so and differentiable through torch.autograd.

    h = layer_norm(features, w, b)                       # features before the encoding
    angles = linear(h, W, bias, activation="tanh")       # features -> angles
    E = VQCFunction.apply(circ, params, angles)
    logits = linear(E, V, c)                             # read-out
    s = log_probs(logits, labels, top=3)                 # s.logp, s.entropy, s.top_logp, ...
    (-s.logp.mean()).backward()

To serve a trained model, with its weights in 8 bits and outcomes that a cheaper one drafted:

    V8 = quantize(V)                                     # once
    logits = linear_quantized(E, V8, c)                  # [sequences, drafts + 1, outcomes]
    v = verify_drafts(logits, draft_logits, drafted, uniforms)     # v.outcomes, v.accepted

The outcomes may be a circuit's own: its probabilities are weights, and those of a shallower one can
be the draft.  p, r: circ.forward_ex(params, angles, probs=True)[1] of both, [samples, 2^n]:

    v = verify_drafts(p[:, None].expand(-1, k + 1, -1), r[:, None].expand(-1, k, -1), drafted,
                      uniforms, kind="weights")

Tensors are cuda tensors of one type (float32, float16 or bfloat16); statistics and sums are
float32.  Leading dimensions are rows.  Rows may be any distance apart; a row's elements must be
adjacent.  Wrong arguments raise ValueError, a failed call of the library VQCError (in a backward
pass RuntimeError, with the same message).  Derivatives are first ones, of the backward pass:
tangents of forward mode raise ValueError, and going on through a gradient RuntimeError.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import math
import os
from typing import NamedTuple, Optional

import torch

from . import _lib


def _load():
    """The native half (csrc/torch_layers.cpp); there is no other implementation."""
    path = os.path.join(os.path.dirname(_lib.LIB_PATH), "vqc_torch.so")
    if not os.path.exists(path):
        raise RuntimeError(f"extension not built: {path} is missing "
                           "(run `python -m paper_2607_11985_amd.build`)")
    _lib.load()
    loader = importlib.machinery.ExtensionFileLoader("vqc_torch", path)
    module = importlib.util.module_from_spec(
        importlib.util.spec_from_file_location("vqc_torch", path, loader=loader))
    loader.exec_module(module)
    module.set_error_type(_lib.VQCError)
    return module


_ext = _load()
_ACT, _SCORES = _lib.ACT, _lib.SCORES


class LogProbs(NamedTuple):
    """What log_probs returns."""
    logp: torch.Tensor        # log probabilities of the targets, float32, their shape
    entropy: torch.Tensor     # [rows...] float32
    top_logp: torch.Tensor    # [rows..., top] float32, falling
    top_index: torch.Tensor   # [rows..., top] int64


class Quantized(NamedTuple):
    """Rows in 8-bit integers: values * scales[..., None] stand for the numbers."""
    values: torch.Tensor      # [rows..., cols] int8
    scales: torch.Tensor      # [rows...] float32


class Verified(NamedTuple):
    """What verify_drafts returns."""
    outcomes: torch.Tensor    # [sequences..., drafts + 1] int64, -1 behind the last one
    accepted: torch.Tensor    # [sequences...] int64, how many drafts


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the last dimension."""
    return _ext.layer_norm(x, weight, bias, eps)


def linear(x, weight, bias=None, activation: str = "none", residual=None):
    """activation(x weight^T + bias) + residual, activation one of none, relu, gelu, silu, tanh.

    weight [n_out, n_in]; residual of the result's shape."""
    act = _ACT.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(_ACT)}, got {activation!r}")
    return _ext.linear(x, weight, bias, act, residual)


def log_probs(scores, targets: Optional[torch.Tensor] = None, top: int = 0,
              kind: str = "logits", temperature: float = 1.0) -> LogProbs:
    """Log probabilities of the target outcomes, entropy and the `top` most probable outcomes.

    scores [..., outcomes]: logits, or with kind="weights" unnormalised probabilities such as
    those of Circuit.forward_ex (no gradient).  targets [...] or [..., n] int64, -1 for none.
    logp and entropy are differentiable with respect to logits."""
    code = _SCORES.get(kind)
    if code is None:
        raise ValueError(f"kind must be one of {sorted(_SCORES)}, got {kind!r}")
    if not (temperature > 0 and math.isfinite(temperature)):
        raise ValueError(f"temperature must be finite and positive, got {temperature}")
    if code and temperature != 1.0:
        raise ValueError("weights have no temperature")
    return LogProbs(*_ext.log_probs(scores, targets, top, code, 1.0 / temperature))


def quantize(x) -> Quantized:
    """Each row (over the last dimension) in integers of [-127, 127] and the step between them, its
    largest magnitude over 127; values to the nearest integer, ties to even.  No gradient.

    A row with an infinity or a NaN has a step of NaN."""
    return Quantized(*_ext.quantize(x))


def linear_quantized(x, weight: Quantized, bias=None, activation: str = "none", residual=None,
                     dtype: Optional[torch.dtype] = None):
    """linear() for inference with rows and weight in 8-bit integers, summed exactly.

    x [..., n_in]: a tensor, quantised row by row as by quantize(), its type that of bias, residual
    and result; or Quantized, with bias, residual and result of dtype (float32).  weight:
    quantize() of a weight [n_out, n_in], once.  No gradient.

    quantize() starts every row on a multiple of 16 bytes, where the products read it fastest.  Copies
    of its values (clone, contiguous, another device) pack rows whose n_in is no such multiple: the
    results are the same, in up to six times the time.  Quantise on the device that serves."""
    act = _ACT.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(_ACT)}, got {activation!r}")
    w, w_scales = weight
    if isinstance(x, torch.Tensor):
        return _ext.linear_quantized(x, None, w, w_scales, bias, act, residual, dtype)
    q, scales = x
    return _ext.linear_quantized(q, scales, w, w_scales, bias, act, residual, dtype)


def verify_drafts(target, draft, drafted, uniforms, kind: str = "logits",
                  temperature: float = 1.0) -> Verified:
    """Drafted outcomes verified with given uniform numbers, so that what is answered is distributed
    as the target's own outcomes.

    target [..., drafts + 1, outcomes] and draft [..., drafts, outcomes]: the scores that the model
    and the draft gave each position (kind and temperature as for log_probs), draft None where the
    drafts were certain; drafted [..., drafts] int64, the first index that is no outcome, such as
    -1, ending a sequence's drafts; uniforms [..., drafts + 1] float32 or float64 in [0, 1).  The
    outcomes are the accepted drafts, one drawn behind them (-1 from a row without any), then -1.
    With no drafts an outcome of each target row is drawn.  No gradient."""
    code = _SCORES.get(kind)
    if code is None:
        raise ValueError(f"kind must be one of {sorted(_SCORES)}, got {kind!r}")
    if not (temperature > 0 and math.isfinite(temperature) and math.isfinite(1.0 / temperature)):
        raise ValueError(f"temperature must be finite and positive, got {temperature}")
    if code and temperature != 1.0:
        raise ValueError("weights have no temperature")
    return Verified(*_ext.verify_drafts(target, draft, drafted, uniforms, code, 1.0 / temperature))
