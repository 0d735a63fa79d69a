"""Operators of a language model around the SRU layer (argument marshalling
over libsru.so, as in ``sru``): a gated linear recurrence, norms, gate and
residual scale between blocks, log probabilities of tokens and distillation at
the head.

Activations and logits are float32 or bfloat16; parameters, states, statistics
and losses are float32.  Every call checks its tensors, runs on the current
stream, allocates the outputs that ``out`` does not hold and takes a workspace
of its own unless it is given one.
"""

from __future__ import annotations

import torch

from . import sru
from .sru import _check, _req, _ws

DTYPE_FP32, DTYPE_BF16 = 0, 1
MAX_TOP, MAX_TEACHER = 64, 1024
GATE_SILU, GATE_SIGMOID = 0, 1
LRU_STEPS = 8
_INT_MAX = (1 << 31) - 1  # sizes are ints in the library; ctypes would cut larger ones

_CODES = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}


_Tensor = torch.Tensor


def _ptr(t):
    return None if t is None else t.data_ptr()


def _plain(t, shape, dtype, device):
    """Whether t is a contiguous tensor of this kind on a GPU device (one known
    to be so): most arguments pass by this one expression, the others go to the
    checks that name what is wrong.  A small call is bound by the host."""
    return (t.__class__ is _Tensor and t.dtype is dtype and t.shape == shape
            and t.device == device and t.is_contiguous())


def _dtype(t, name):
    """The library's code of t's type."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.dtype not in _CODES:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return _CODES[t.dtype]


def _too_large(t, name):
    return ValueError(f"{name} is too large: {tuple(t.shape)}")


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


def _out(out, name, shape, dtype, like):
    """out[name] if the caller gave it (checked), else a new tensor on the
    device of `like`."""
    t = None if out is None else out.get(name)
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    _req(t, name, shape, dtype=dtype, device=like.device)
    return t


def _out_like(out, name, like):
    """_out for one of the shape and type of the contiguous tensor `like`."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty_like(like)
    _req(t, name, like.shape, dtype=like.dtype, device=like.device)
    return t


def _new_like(like):
    """A new contiguous tensor of the shape and type of `like`."""
    return torch.empty_like(like) if like.is_contiguous() else like.new_empty(like.shape)


def _logits(logits, temperature):
    """(code, N, V, device, pitch) of checked logits."""
    code = _dtype(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be a 2-d tensor [N, V]")
    dv = _here(logits, "logits")
    if not 0.0 < temperature < float("inf"):
        raise ValueError(f"temperature must be positive and finite, got {temperature}")
    N, V = logits.shape
    if N > _INT_MAX or V > _INT_MAX:
        raise _too_large(logits, "logits")
    return code, N, V, dv, _pitch(logits, "logits", (N, V), logits.dtype, dv)


def _dlogits(dlogits, logits, dv):
    """(dlogits, its pitch): the caller's, which may be the logits, or new."""
    if dlogits is None:
        dlogits = _new_like(logits)
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
    if not 0 <= top <= MAX_TOP:
        raise ValueError(f"top must be 0 .. {MAX_TOP}, got {top}")
    o = dict(logprob=_out(out, "logprob", (N,), _F32, logits),
             entropy=_out(out, "entropy", (N,), _F32, logits),
             stats=_out(out, "stats", (N, 2), _F32, logits),
             top_ids=_out(out, "top_ids", (N, top), _I64, logits) if top else None,
             top_logprobs=_out(out, "top_logprobs", (N, top), _F32, logits) if top else None)
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
    if K > _INT_MAX:
        raise _too_large(teacher_logits, "teacher_logits")
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
    o = dict(loss=_out(out, "loss", (N,), _F32, logits), stats=_out(out, "stats", (N, 2), _F32, logits))
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
    o = dict(loss=_out(out, "loss", (N,), _F32, logits), stats=_out(out, "stats", (N, 2), _F32, logits))
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


def _row_pitch(t, name, shape, dtype, device):
    """The distance of consecutive rows of a [..., d] tensor (None: 0)."""
    if t is None:
        return 0
    if _plain(t, shape, dtype, device):
        return shape[-1]
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
    # leading dimensions of more than one row, from the last: one pitch for all
    ld, span = None, 1
    for n, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n > 1:
            if ld is None:
                ld = step
            elif step != ld * span:
                raise ValueError(f"{name} must have rows at equal distances")
            span *= n
    d = shape[-1]
    if (d > 1 and t.stride(-1) != 1) or (ld is not None and ld < d):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return d if ld is None else ld


def _norm_inputs(x, y, z, w_post, scale, w_pre, dtype=None):
    """Checked inputs: M, d, activation type (dtype, where there is no y to have
    it), its code, residual code, device, and the pitches of x, y and z."""
    res = _dtype(x, "x")
    if x.dim() < 1:
        raise ValueError("x must have a last dimension")
    dv = _here(x, "x")
    shape = x.shape
    d = shape[-1]
    if y is None:
        if w_pre is None or w_post is not None or z is not None or scale is not None:
            raise ValueError("without y there is only the norm of x: give w_pre alone")
        act = x.dtype if dtype is None else dtype
        code = _CODES.get(act)
    else:
        act, code = y.dtype if isinstance(y, torch.Tensor) else None, _dtype(y, "y")
    if x.dtype != act and (x.dtype != _F32 or code is None):
        raise ValueError(f"x must be {act} or float32 beside bfloat16, got {x.dtype}")
    pitch = (_row_pitch(x, "x", shape, x.dtype, dv), _row_pitch(y, "y", shape, act, dv),
             _row_pitch(z, "z", shape, act, dv))
    for n, w in (("w_post", w_post), ("scale", scale), ("w_pre", w_pre)):
        if w is not None and not _plain(w, (d,), _F32, dv):
            _req(w, n, (d,), device=dv)
    M = x.numel() // d if d else 0
    if M > _INT_MAX or d > _INT_MAX:
        raise _too_large(x, "x")
    return M, d, act, code, res, dv, pitch


def _row_out(out, name, like, dtype=None):
    """(out[name] or a new tensor, of the shape and type of `like` (or of type
    dtype); its row pitch)."""
    t = None if out is None else out.get(name)
    if dtype is None:
        dtype = like.dtype
    if t is not None:
        return t, _row_pitch(t, name, like.shape, dtype, like.device)
    t = _new_like(like) if dtype is like.dtype else like.new_empty(like.shape, dtype=dtype)
    return t, like.shape[-1]


def residual_norm_forward(x, y=None, w_post=None, z=None, scale=None, w_pre=None,
                          gate=GATE_SILU, eps=1e-6, out=None, dtype=None):
    """Between two blocks: dict(x_out, o, rstd) with

        x_out = x + scale * (y rstd(y) w_post) * gate(z)
        o     = x_out rstd(x_out) w_pre,      rstd(v) = 1 / sqrt(mean(v^2) + eps)

    over the last dimension.  x is the residual stream [..., d], y the block's
    output, z the gate's input (z sigma(z), or sigma(z) with GATE_SIGMOID);
    w_post, scale and w_pre are float32 [d].  Each of w_post, z, scale and w_pre
    may be None (no norm of y, no gate, scale 1, no o); without y, o is the norm
    of x.  x may be float32 beside bfloat16 activations; the type of o is y's, or
    without y `dtype` (None: x's).  Rows may be strided (slices of a projection).
    out may hold x_out (x itself), o and rstd."""
    M, d, act, code, res, dv, (ldx, ldy, ldz) = _norm_inputs(x, y, z, w_post, scale, w_pre, dtype)
    if dtype is not None and dtype != act:
        raise ValueError(f"y is {act}, and so is o: not {dtype}")
    x_out, o, ldxo, ldo = None, None, 0, 0
    if y is not None:
        x_out, ldxo = _row_out(out, "x_out", x)
    if w_pre is not None:
        o, ldo = _row_out(out, "o", x if y is None else y, act)
    rstd = _out(out, "rstd", (*x.shape[:-1], 2), _F32, x)
    st = sru.lib().sru_residual_norm_forward(M, d, code, res, gate, eps, _ptr(x), ldx, _ptr(y),
                                             ldy, _ptr(z), ldz, _ptr(w_post), _ptr(scale),
                                             _ptr(w_pre), _ptr(x_out), ldxo, _ptr(o), ldo,
                                             _ptr(rstd), sru._stream())
    _check(st, "sru_residual_norm_forward")
    return dict(x_out=x_out, o=o, rstd=rstd)


def residual_norm_backward(x, y, rstd, dx_out=None, do=None, w_post=None, z=None, scale=None,
                           w_pre=None, gate=GATE_SILU, eps=1e-6, out=None, ws=None):
    """Gradients of residual_norm_forward, given its inputs, its rstd (which
    holds eps) and the gradients of x_out and o (None: zeros; do has the type of
    o): dict(dx, dy, dz, dw_post, dscale, dw_pre), None where the input was.  out
    may hold any of them (dx may be dx_out itself, dy and dz slices of a larger
    tensor)."""
    M, d, act, code, res, dv, (ldx, ldy, ldz) = _norm_inputs(
        x, y, z, w_post, scale, w_pre, do.dtype if isinstance(do, torch.Tensor) else None)
    shape = x.shape
    _req(rstd, "rstd", tuple(shape[:-1]) + (2,), device=dv)
    lddxo = _row_pitch(dx_out, "dx_out", shape, x.dtype, dv)
    lddo = _row_pitch(do, "do", shape, act, dv)
    g = {}
    g["dx"], lddx = _row_out(out, "dx", x)
    g["dy"], lddy = _row_out(out, "dy", y) if y is not None else (None, 0)
    g["dz"], lddz = _row_out(out, "dz", z) if z is not None else (None, 0)
    for n, w in (("dw_post", w_post), ("dscale", scale), ("dw_pre", w_pre)):
        g[n] = None if w is None else _out_like(out, n, w)
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_residual_norm_backward_workspace_bytes(M, d), dv)
    st = lib.sru_residual_norm_backward(
        M, d, code, res, gate, _ptr(x), ldx, _ptr(y), ldy, _ptr(z), ldz, _ptr(w_post),
        _ptr(scale), _ptr(w_pre), _ptr(rstd), _ptr(dx_out), lddxo, _ptr(do), lddo, _ptr(g["dx"]),
        lddx, _ptr(g["dy"]), lddy, _ptr(g["dz"]), lddz, _ptr(g["dw_post"]), _ptr(g["dscale"]),
        _ptr(g["dw_pre"]), _ptr(ws), nbytes, sru._stream())
    _check(st, "sru_residual_norm_backward")
    return g


def _seq(t, name, shape, dtype, device):
    """The distances of consecutive steps and of sequences of a [L, B, d]
    tensor with contiguous features."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if not (t.is_cuda or sru._on_gpu(t)):
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    st, sb, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have contiguous features")
    return st, sb


def _lru_inputs(x, r, i, lam, mask, reset):
    """Checked inputs: (L, B, d), code, device, and the distances of x, r, i."""
    code = _dtype(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be a 3-d tensor [L, B, d]")
    dv = _here(x, "x")
    shape = x.shape
    L, B, d = shape
    if L > _INT_MAX or B > _INT_MAX or d > _INT_MAX:
        raise _too_large(x, "x")
    steps = (_seq(x, "x", shape, x.dtype, dv), _seq(r, "r", shape, x.dtype, dv),
             _seq(i, "i", shape, x.dtype, dv))
    _req(lam, "lam", (d,), device=dv)
    if mask is not None:
        _req(mask, "mask", (L, B), dtype=torch.uint8, device=dv)
    if reset is not None:
        _req(reset, "reset", (L, B), dtype=torch.uint8, device=dv)
    return shape, code, dv, steps


def _seq_out(out, name, like):
    """(out[name] or a new tensor, of the shape and type of `like`; its
    distances)."""
    t = None if out is None else out.get(name)
    if t is None:
        _, B, d = like.shape
        return _new_like(like), (B * d, d)
    return t, _seq(t, name, like.shape, like.dtype, like.device)


def lru_forward(x, r, i, lam, h0=None, mask=None, reset=None, c=8.0, keep_states=True, out=None,
                ws=None):
    """Gated linear recurrence over the first dimension of x, r, i [L, B, d]:

        a = exp(-c softplus(lam) sigma(r)),  h_t = a h_{t-1} + sqrt(1 - a^2) sigma(i) x

    lam [d]; h0 [B, d] float32 (None: zeros); mask [L, B] uint8, nonzero where a
    step is padded (the state passes, the output is 0); reset [L, B] uint8,
    nonzero where a new document starts (a = 0).  Returns dict(H [L, B, d],
    h_last [B, d], states): states, the state before every LRU_STEPS-th step,
    is what lru_backward needs (None with keep_states=False).  x, r, i and H
    may be strided: slices of one projection, or [B, L, d] transposed.  out may
    hold H, h_last (h0 itself: the state taken on in place) and states."""
    shape, code, dv, (sx, sr, si) = _lru_inputs(x, r, i, lam, mask, reset)
    L, B, d = shape
    _req(h0, "h0", (B, d), optional=True, device=dv)
    H, sh = _seq_out(out, "H", x)
    h_last = _out(out, "h_last", (B, d), _F32, x)
    states = _out(out, "states", (-(-L // LRU_STEPS), B, d), _F32, x) if keep_states else None
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_lru_forward_workspace_bytes(L, B, d), dv)
    st = lib.sru_lru_forward(L, B, d, code, _ptr(x), *sx, _ptr(r), *sr, _ptr(i), *si, _ptr(lam), c,
                             _ptr(h0), _ptr(mask), _ptr(reset), _ptr(H), *sh, _ptr(h_last),
                             _ptr(states), _ptr(ws), nbytes, sru._stream())
    _check(st, "sru_lru_forward")
    return dict(H=H, h_last=h_last, states=states)


def lru_backward(x, r, i, lam, states, dH, dh_last=None, mask=None, reset=None, c=8.0,
                 want_dh0=True, out=None, ws=None):
    """Gradients of lru_forward given its inputs, its states and the gradients
    dH [L, B, d] of H and dh_last [B, d] of h_last: dict(dx, dr, di, dlam, dh0).
    out may hold any of them (dx, dr, di as slices of one tensor)."""
    shape, code, dv, (sx, sr, si) = _lru_inputs(x, r, i, lam, mask, reset)
    L, B, d = shape
    _req(states, "states", (-(-L // LRU_STEPS), B, d), device=dv)
    sdh = _seq(dH, "dH", shape, x.dtype, dv)
    _req(dh_last, "dh_last", (B, d), optional=True, device=dv)
    dx, sdx = _seq_out(out, "dx", x)
    dr, sdr = _seq_out(out, "dr", x)
    di, sdi = _seq_out(out, "di", x)
    dlam = _out_like(out, "dlam", lam)
    dh0 = _out(out, "dh0", (B, d), _F32, x) if want_dh0 else None
    lib = sru.lib()
    ws, nbytes = _ws(ws, lib.sru_lru_backward_workspace_bytes(L, B, d), dv)
    st = lib.sru_lru_backward(L, B, d, code, _ptr(x), *sx, _ptr(r), *sr, _ptr(i), *si, _ptr(lam),
                              c, _ptr(states), _ptr(dH), *sdh, _ptr(dh_last), _ptr(mask),
                              _ptr(reset), _ptr(dx), *sdx, _ptr(dr), *sdr, _ptr(di), *sdi,
                              _ptr(dlam), _ptr(dh0), _ptr(ws), nbytes, sru._stream())
    _check(st, "sru_lru_backward")
    return dict(dx=dx, dr=dr, di=di, dlam=dlam, dh0=dh0)


def _step_rows(t, name, shape, dtype, device):
    """The distance of sequences of a [B, d] tensor with contiguous features."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-d tensor [B, d]")
    return _seq(t.unsqueeze(0), name, (1,) + tuple(shape), dtype, device)[1]


def lru_step(x, r, i, lam, h, c=8.0, out=None, mask=None, reset=None):
    """One token of the recurrence: x, r, i [B, d], the state h [B, d] float32
    taken on in place.  mask and reset [B] uint8 as in lru_forward: a stream
    without a token (its state stays, its output is 0), one that starts a new
    document.  Returns the output [B, d] (out, or a new tensor)."""
    code = _dtype(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be a 2-d tensor [B, d]")
    dv, dt, shape = _here(x, "x"), x.dtype, x.shape
    B, d = shape
    if B > _INT_MAX or d > _INT_MAX:
        raise _too_large(x, "x")
    fast = x.stride(1) == 1
    for n, t in (("r", r), ("i", i)):
        fast = (fast and t.__class__ is torch.Tensor and t.dtype is dt and t.shape == shape
                and t.device == dv and t.stride(1) == 1)
    if not fast:  # one by one, for the message
        for n, t in (("x", x), ("r", r), ("i", i)):
            _step_rows(t, n, shape, dt, dv)
    if not (_plain(lam, (d,), _F32, dv) and _plain(h, shape, _F32, dv)):
        _req(lam, "lam", (d,), device=dv)
        _req(h, "h", (B, d), device=dv)
    if mask is not None:
        _req(mask, "mask", (B,), dtype=torch.uint8, device=dv)
    if reset is not None:
        _req(reset, "reset", (B,), dtype=torch.uint8, device=dv)
    if out is None:
        out, so = _new_like(x), d
    else:
        so = _step_rows(out, "out", shape, dt, dv)
    hp = _ptr(h)
    st = sru.lib().sru_lru_forward(1, B, d, code, _ptr(x), 0, x.stride(0), _ptr(r), 0,
                                   r.stride(0), _ptr(i), 0, i.stride(0), _ptr(lam), c, hp,
                                   _ptr(mask), _ptr(reset), _ptr(out), 0, so, hp, None, None, 0,
                                   sru._stream())
    _check(st, "sru_lru_forward")
    return out
