"""Operators of a language model around the SRU layer (argument marshalling
over libsru.so, as in ``sru``): log probabilities of tokens and distillation at
its head.

Activations and logits are float32 or bfloat16; parameters, states, statistics
and losses are float32.  Every call checks its tensors, runs on the current
stream, allocates the outputs that ``out`` does not hold and takes a workspace
of its own unless it is given one.
"""

from __future__ import annotations

import torch

from . import sru
from .sru import _check, _ptr, _req, _ws

DTYPE_FP32, DTYPE_BF16 = 0, 1
MAX_TOP, MAX_TEACHER = 64, 1024

_CODES = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}


def _dtype(t, name):
    """The library's code of t's type."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.dtype not in _CODES:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return _CODES[t.dtype]


def _here(t, name):
    """The device of t, which must be the current one: the call runs on its
    current stream."""
    if not sru._on_gpu(t):
        raise ValueError(f"{name} must be a GPU tensor")
    if t.is_cuda and t.device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    return t.device


def _pitch(t, name, shape, dtype, device):
    """The row pitch of a [N, V] tensor whose rows are contiguous and apart."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if not sru._on_gpu(t):
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    n, v = shape
    ld = max(v, 1) if n <= 1 else t.stride(0)
    if (v > 1 and t.stride(1) != 1) or ld < v:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return ld


def _out(out, name, shape, dtype, device):
    """out[name] if the caller gave it (checked), else a new tensor."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _req(t, name, shape, dtype=dtype, device=device)
    return t


def _logits(logits, temperature):
    """(code, N, V, device, pitch) of checked logits."""
    code = _dtype(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be a 2-d tensor [N, V]")
    dv = _here(logits, "logits")
    if not 0.0 < temperature < float("inf"):
        raise ValueError(f"temperature must be positive and finite, got {temperature}")
    N, V = logits.shape
    return code, N, V, dv, _pitch(logits, "logits", (N, V), logits.dtype, dv)


def _dlogits(dlogits, logits, dv):
    """(dlogits, its pitch): the caller's, which may be the logits, or new."""
    if dlogits is None:
        dlogits = torch.empty(tuple(logits.shape), dtype=logits.dtype, device=dv)
    return dlogits, _pitch(dlogits, "dlogits", logits.shape, logits.dtype, dv)


_F32, _I64 = torch.float32, torch.int64


def token_logprobs(logits, tokens, top=0, temperature=1.0, out=None, ws=None):
    """Log probabilities of one given token per row of logits [N, V].

    tokens [N] int64 (one outside 0 .. V-1: the row is not scored, 0); top:
    how many of the best alternatives to return (up to MAX_TOP).  Returns
    dict(logprob [N], entropy [N], stats [N, 2], top_ids [N, top] int64,
    top_logprobs [N, top]), the last two None without alternatives.  Rows may
    be strided; logits of -inf are tokens that are not possible."""
    code, N, V, dv, ld = _logits(logits, temperature)
    _req(tokens, "tokens", (N,), dtype=_I64, device=dv)
    o = dict(logprob=_out(out, "logprob", (N,), _F32, dv),
             entropy=_out(out, "entropy", (N,), _F32, dv),
             stats=_out(out, "stats", (N, 2), _F32, dv),
             top_ids=_out(out, "top_ids", (N, top), _I64, dv) if top else None,
             top_logprobs=_out(out, "top_logprobs", (N, top), _F32, dv) if top else None)
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_token_logprobs_workspace_bytes(N, V, code, top), dv)
    st = lib.sru_token_logprobs(_ptr(logits), ld, code, _ptr(tokens), N, V, top, temperature,
                                _ptr(o["logprob"]), _ptr(o["entropy"]), _ptr(o["stats"]),
                                _ptr(o["top_ids"]), _ptr(o["top_logprobs"]), _ptr(ws), nbytes,
                                sru._stream())
    _check(st, "sru_token_logprobs")
    return o


def token_logprobs_backward(logits, tokens, fw, dlogprob=None, dentropy=None, dtop=None,
                            temperature=1.0, dlogits=None):
    """Gradient of token_logprobs with respect to the logits.

    fw: what token_logprobs returned for the same arguments; dlogprob [N],
    dentropy [N] and dtop [N, top] are the gradients of its results (None: no
    gradient).  Writes dlogits, which may be the logits themselves, or a new
    tensor."""
    code, N, V, dv, ld = _logits(logits, temperature)
    _req(tokens, "tokens", (N,), dtype=_I64, device=dv)
    _req(fw["stats"], "stats", (N, 2), device=dv)
    _req(dlogprob, "dlogprob", (N,), optional=True, device=dv)
    _req(dentropy, "dentropy", (N,), optional=True, device=dv)
    entropy, top_ids, top = None, None, 0
    if dentropy is not None:
        entropy = fw["entropy"]
        _req(entropy, "entropy", (N,), device=dv)
    if dtop is not None:
        top_ids = fw["top_ids"]
        if not isinstance(top_ids, torch.Tensor) or top_ids.dim() != 2:
            raise ValueError("dtop needs the top_ids [N, top] of the forward call")
        top = top_ids.shape[1]
        _req(top_ids, "top_ids", (N, top), dtype=_I64, device=dv)
        _req(dtop, "dtop", (N, top), device=dv)
    dlogits, ldd = _dlogits(dlogits, logits, dv)
    st = sru.lib().sru_token_logprobs_backward(
        _ptr(logits), ld, code, _ptr(tokens), _ptr(fw["stats"]), _ptr(entropy), _ptr(dlogprob),
        _ptr(dentropy), _ptr(top_ids), _ptr(dtop), N, V, top, temperature, _ptr(dlogits), ldd,
        sru._stream())
    _check(st, "sru_token_logprobs_backward")
    return dlogits


def _teacher(teacher_ids, teacher_logits, N, dv):
    """(code, K) of checked teacher entries."""
    code = _dtype(teacher_logits, "teacher_logits")
    if teacher_logits.dim() != 2:
        raise ValueError("teacher_logits must be a 2-d tensor [N, K]")
    K = teacher_logits.shape[1]
    _req(teacher_ids, "teacher_ids", (N, K), dtype=_I64, device=dv)
    _req(teacher_logits, "teacher_logits", (N, K), dtype=teacher_logits.dtype, device=dv)
    return code, K


def distill_forward(logits, teacher_ids, teacher_logits, temperature=1.0, out=None, ws=None):
    """KL divergence of the student's softmax(logits / T) from the teacher's
    over its K best tokens, per row: dict(loss [N], stats [N, 2]).

    teacher_ids [N, K] int64 and teacher_logits [N, K]; an entry with an id
    outside 0 .. V-1 or a logit of -inf is not kept, and the kept ones are
    normalised among themselves.  A row without any has loss 0."""
    code, N, V, dv, ld = _logits(logits, temperature)
    tcode, K = _teacher(teacher_ids, teacher_logits, N, dv)
    o = dict(loss=_out(out, "loss", (N,), _F32, dv), stats=_out(out, "stats", (N, 2), _F32, dv))
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_distill_workspace_bytes(N, V, code), dv)
    st = lib.sru_distill_forward(_ptr(logits), ld, code, _ptr(teacher_ids), _ptr(teacher_logits),
                                 tcode, N, V, K, temperature, _ptr(o["loss"]), _ptr(o["stats"]),
                                 _ptr(ws), nbytes, sru._stream())
    _check(st, "sru_distill_forward")
    return o


def distill_backward(logits, teacher_ids, teacher_logits, stats, dloss, temperature=1.0,
                     dlogits=None):
    """Gradient of distill_forward with respect to the logits, given the
    gradient dloss [N] of its losses.  Writes dlogits, which may be the logits
    themselves, or a new tensor."""
    code, N, V, dv, ld = _logits(logits, temperature)
    tcode, K = _teacher(teacher_ids, teacher_logits, N, dv)
    _req(stats, "stats", (N, 2), device=dv)
    _req(dloss, "dloss", (N,), device=dv)
    dlogits, ldd = _dlogits(dlogits, logits, dv)
    st = sru.lib().sru_distill_backward(_ptr(logits), ld, code, _ptr(teacher_ids),
                                        _ptr(teacher_logits), tcode, _ptr(stats), _ptr(dloss), N,
                                        V, K, temperature, _ptr(dlogits), ldd, sru._stream())
    _check(st, "sru_distill_backward")
    return dlogits


def distill_forward_backward(logits, teacher_ids, teacher_logits, dloss, temperature=1.0,
                             dlogits=None, out=None, ws=None):
    """distill_forward and distill_backward in one call, for row weights dloss
    [N] that are known beforehand: dict(loss, stats, dlogits)."""
    code, N, V, dv, ld = _logits(logits, temperature)
    tcode, K = _teacher(teacher_ids, teacher_logits, N, dv)
    _req(dloss, "dloss", (N,), device=dv)
    o = dict(loss=_out(out, "loss", (N,), _F32, dv), stats=_out(out, "stats", (N, 2), _F32, dv))
    o["dlogits"], ldd = _dlogits(dlogits, logits, dv)
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_distill_workspace_bytes(N, V, code), dv)
    st = lib.sru_distill_forward_backward(_ptr(logits), ld, code, _ptr(teacher_ids),
                                          _ptr(teacher_logits), tcode, _ptr(dloss), N, V, K,
                                          temperature, _ptr(o["loss"]), _ptr(o["stats"]),
                                          _ptr(o["dlogits"]), ldd, _ptr(ws), nbytes,
                                          sru._stream())
    _check(st, "sru_distill_forward_backward")
    return o
