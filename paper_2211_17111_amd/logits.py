"""Logits operators of libbevpool.so (include/bevpool_logits.h): log
probabilities of tokens with entropy and top alternatives, and distillation from
a teacher's alternatives.

A row of logits x (a vocabulary, or a pixel's depth bins) stands for the
distribution softmax(scale * x).  ``*_forward`` and ``*_backward`` allocate their
outputs and launch the kernels; ``logprobs`` and ``distill`` are their
differentiable forms.  What a teacher answers is what a student learns from:

    answer = logprobs_forward(teacher_logits, k=32, scale=scale)
    loss = distill(student_logits, answer.top_ids, answer.top, scale).mean()

and where the gradient of every row's loss is known beforehand, ``distill_step``
gives loss and gradient in one call, with the logits read once.

Ids outside [0, V) are dropped: a position without a token has log probability 0
and no gradient, an alternative without an id no part in the loss.  A logit of
-inf has probability 0; a row of nothing else has no distribution (log
probabilities -inf, entropy 0, gradient 0).

Conventions of tensors, streams and captures are those of ``rows``: matrices may
have any distance between their rows, nothing synchronises, everything runs on
the current stream of the tensors' device or on ``stream``.
"""

from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import bevpool as _bp
from .rows import (_DTYPE_CODE, _F32, _I32, _KEY_CODE, _LIMIT, _dense, _device, _elsewhere, _i32, _i64, _int,
                   _matrix, _stream, _sz, _vp)

_f32 = ctypes.c_float
_size_args = [_i64, _i64, _i32, _int, ctypes.POINTER(_sz)]
_rows_args = [_i64, _i64, _i32, _int]                  # rows, V, k, dtype
_logits_args = [_vp, _i64, _f32, _int, _vp]            # logits, stride, scale, key type, ids
_ARGTYPES = {
    "bevpool_logprobs_workspace_size": _size_args,
    "bevpool_logprobs_forward": _rows_args + _logits_args + [_vp] * 7 + [_sz, _vp],
    "bevpool_logprobs_backward": _rows_args + _logits_args + [_vp] * 9,
    "bevpool_distill_workspace_size": _size_args,
    "bevpool_distill_forward": _rows_args + _logits_args + [_vp, _int, _vp, _vp, _vp, _sz, _vp],
    "bevpool_distill_backward": _rows_args + [_vp] + _logits_args + [_vp, _int, _vp, _vp, _vp],
    "bevpool_distill_step": _rows_args + [_vp] + _logits_args + [_vp, _int, _vp, _vp, _vp, _vp, _sz, _vp],
}

_lib = None


def load_library() -> ctypes.CDLL:
    """libbevpool.so with the logits operators' signatures (raises if it has not been built)."""
    global _lib
    if _lib is None:
        lib = _bp.load_library()
        for name, argtypes in _ARGTYPES.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = _int, argtypes
        _lib = lib
    return _lib


def _call(name: str, *args) -> None:
    lib = _lib or load_library()
    status = getattr(lib, name)(*args)
    if status != 0:
        _bp._check(lib, status, name)


_sizes: dict = {}


def _workspace(name: str, args, dev: torch.device):
    """(tensor that must live until the launch, its address, its bytes)."""
    nbytes = _sizes.get((name, args))
    if nbytes is None:
        n = _sz(0)
        _call(name, *args, ctypes.byref(n))
        if len(_sizes) >= 1024:
            _sizes.clear()
        nbytes = _sizes[name, args] = n.value
    if nbytes == 0:
        return None, None, 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    return ws, ws.data_ptr(), nbytes


def _check_count(k: int) -> None:
    if not 0 <= k < _LIMIT:  # (a larger one would pass its low 32 bits only)
        raise ValueError(f"k = {k} is negative or exceeds 2^31 - 1")


# --------------------------------------------------------- log probabilities

@dataclass
class Logprobs:
    """Of every row: ``logprob`` of its given token (None where none were
    given), ``lse`` the log of the sum of e^(scale x), ``entropy`` (None unless
    asked for), ``top`` and ``top_ids`` (T, k) the best alternatives' log
    probabilities and ids, -inf and -1 where fewer have a probability (None
    for k = 0).  ``stats`` (T, 2): the largest logit and the sum of
    e^(scale (x - largest)), which the gradient is formed from."""
    logprob: torch.Tensor | None
    lse: torch.Tensor
    entropy: torch.Tensor | None
    top: torch.Tensor | None
    top_ids: torch.Tensor | None
    stats: torch.Tensor


def logprobs_forward(logits: torch.Tensor, ids: torch.Tensor | None = None, k: int = 0, scale: float = 1.0,
                     entropy: bool = False, stream=None) -> Logprobs:
    """Log probabilities under softmax(scale * logits), logits (T, V): of the
    given token ids (T,) int32 or int64, of the k <= 64 best tokens (equal logits
    by index), and the distributions' entropies; all float32."""
    dev = _device(logits, "logits")
    stride = _matrix(logits, "logits", dev)
    T, V = logits.shape
    _check_count(k)
    if ids is not None:
        _dense(ids, "ids", dev, _KEY_CODE, (T,))
    ctx = _elsewhere(dev, stream, logits, ids)
    if ctx is not None:
        with ctx:
            return logprobs_forward(logits, ids, k, scale, entropy)
    f32, code = torch.float32, _DTYPE_CODE[logits.dtype]
    stats = torch.empty((T, 2), dtype=f32, device=dev)
    lse = torch.empty(T, dtype=f32, device=dev)
    logprob = ids_at = logprob_at = h = h_at = top = top_at = top_ids = top_ids_at = None
    key_type = 0
    if ids is not None:
        logprob = torch.empty(T, dtype=f32, device=dev)
        key_type, ids_at, logprob_at = _KEY_CODE[ids.dtype], ids.data_ptr(), logprob.data_ptr()
    if entropy:
        h = torch.empty(T, dtype=f32, device=dev)
        h_at = h.data_ptr()
    if k:
        top = torch.empty((T, k), dtype=f32, device=dev)
        top_ids = torch.empty((T, k), dtype=torch.int32, device=dev)
        top_at, top_ids_at = top.data_ptr(), top_ids.data_ptr()
    ws, ws_at, nbytes = _workspace("bevpool_logprobs_workspace_size", (T, V, k, code), dev)
    _call("bevpool_logprobs_forward", T, V, k, code, logits.data_ptr(), stride, scale, key_type, ids_at,
          stats.data_ptr(), logprob_at, lse.data_ptr(), h_at, top_at, top_ids_at, ws_at, nbytes, _stream(dev))
    return Logprobs(logprob, lse, h, top, top_ids, stats)


def logprobs_backward(logits: torch.Tensor, result: Logprobs, ids: torch.Tensor | None = None, scale: float = 1.0,
                      grad_logprob=None, grad_lse=None, grad_entropy=None, grad_top=None, stream=None) -> torch.Tensor:
    """Gradient (T, V) of the logits, in their type, from the outgoing gradients
    (float32, None for none) of what logprobs_forward returned with the same
    ids and scale."""
    dev = _device(logits, "logits")
    stride = _matrix(logits, "logits", dev)
    T, V = logits.shape
    _dense(result.stats, "stats", dev, _F32, (T, 2))
    key_type, k = 0, 0
    ids_at = entropy_at = top_ids_at = None
    if grad_logprob is not None:
        if ids is None:
            raise ValueError("grad_logprob needs the ids")
        _dense(ids, "ids", dev, _KEY_CODE, (T,))
        _dense(grad_logprob, "grad_logprob", dev, _F32, (T,))
        key_type, ids_at = _KEY_CODE[ids.dtype], ids.data_ptr()
    if grad_lse is not None:
        _dense(grad_lse, "grad_lse", dev, _F32, (T,))
    if grad_entropy is not None:
        if result.entropy is None:
            raise ValueError("grad_entropy needs the entropy of the forward")
        _dense(result.entropy, "entropy", dev, _F32, (T,))
        _dense(grad_entropy, "grad_entropy", dev, _F32, (T,))
        entropy_at = result.entropy.data_ptr()
    if grad_top is not None:
        if result.top_ids is None:
            raise ValueError("grad_top needs the alternatives of the forward")
        if result.top_ids.dim() != 2 or result.top_ids.shape[0] != T:
            raise ValueError(f"top_ids must be ({T}, k), got {tuple(result.top_ids.shape)}")
        k = result.top_ids.shape[1]
        _check_count(k)
        _dense(result.top_ids, "top_ids", dev, _I32, (T, k))
        _dense(grad_top, "grad_top", dev, _F32, (T, k))
        top_ids_at = result.top_ids.data_ptr()
    ctx = _elsewhere(dev, stream, logits, ids, result.stats, result.entropy, result.top_ids, grad_logprob, grad_lse,
                     grad_entropy, grad_top)
    if ctx is not None:
        with ctx:
            return logprobs_backward(logits, result, ids, scale, grad_logprob, grad_lse, grad_entropy, grad_top)
    grad = torch.empty((T, V), dtype=logits.dtype, device=dev)
    _call("bevpool_logprobs_backward", T, V, k, _DTYPE_CODE[logits.dtype], logits.data_ptr(), stride, scale, key_type,
          ids_at, result.stats.data_ptr(), entropy_at, top_ids_at, _bp._ptr(grad_logprob), _bp._ptr(grad_lse),
          _bp._ptr(grad_entropy), _bp._ptr(grad_top), grad.data_ptr(), _stream(dev))
    return grad


# -------------------------------------------------------------- distillation

def _check_distill(logits, ids, teacher, scale: float, renormalise: bool):
    """Checks the inputs of a distillation: (device, (rows, V, k, type), the arguments after them)."""
    dev = _device(logits, "logits")
    stride = _matrix(logits, "logits", dev)
    T, V = logits.shape
    _dense(ids, "ids", dev, _KEY_CODE)
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError(f"ids must be ({T}, k), got {tuple(ids.shape)}")
    k = ids.shape[1]
    _check_count(k)
    _dense(teacher, "teacher", dev, _F32, (T, k))
    return dev, (T, V, k, _DTYPE_CODE[logits.dtype]), (logits.data_ptr(), stride, scale, _KEY_CODE[ids.dtype],
                                                       ids.data_ptr(), teacher.data_ptr(), int(renormalise))


def distill_forward(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, scale: float = 1.0,
                    renormalise: bool = True, stream=None):
    """(loss, stats): of every row of logits (T, V) the divergence
    sum_j q_j (log q_j - log p_j) of p = softmax(scale * logits) from a teacher's
    k <= 256 alternatives: ids (T, k) int32 or int64, teacher (T, k) float32 their
    log probabilities, log q (``renormalise``: their softmax)."""
    dev, sizes, args = _check_distill(logits, ids, teacher, scale, renormalise)
    ctx = _elsewhere(dev, stream, logits, ids, teacher)
    if ctx is not None:
        with ctx:
            return distill_forward(logits, ids, teacher, scale, renormalise)
    T = sizes[0]
    loss = torch.empty(T, dtype=torch.float32, device=dev)
    stats = torch.empty((T, 2), dtype=torch.float32, device=dev)
    ws, ws_at, nbytes = _workspace("bevpool_distill_workspace_size", sizes, dev)
    _call("bevpool_distill_forward", *sizes, *args, loss.data_ptr(), stats.data_ptr(), ws_at, nbytes, _stream(dev))
    return loss, stats


def distill_backward(grad_loss: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor,
                     stats: torch.Tensor, scale: float = 1.0, renormalise: bool = True, stream=None) -> torch.Tensor:
    """Gradient (T, V) of the logits, in their type, from that of the rows' losses."""
    dev, sizes, args = _check_distill(logits, ids, teacher, scale, renormalise)
    T, V = sizes[:2]
    _dense(grad_loss, "grad_loss", dev, _F32, (T,))
    _dense(stats, "stats", dev, _F32, (T, 2))
    ctx = _elsewhere(dev, stream, grad_loss, logits, ids, teacher, stats)
    if ctx is not None:
        with ctx:
            return distill_backward(grad_loss, logits, ids, teacher, stats, scale, renormalise)
    grad = torch.empty((T, V), dtype=logits.dtype, device=dev)
    _call("bevpool_distill_backward", *sizes, grad_loss.data_ptr(), *args, stats.data_ptr(), grad.data_ptr(),
          _stream(dev))
    return grad


def distill_step(grad_loss: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor,
                 scale: float = 1.0, renormalise: bool = True, stream=None):
    """(loss, gradient of the logits): distill_forward and distill_backward in
    one call, where the gradient of the rows' losses is known beforehand."""
    dev, sizes, args = _check_distill(logits, ids, teacher, scale, renormalise)
    T, V = sizes[:2]
    _dense(grad_loss, "grad_loss", dev, _F32, (T,))
    ctx = _elsewhere(dev, stream, grad_loss, logits, ids, teacher)
    if ctx is not None:
        with ctx:
            return distill_step(grad_loss, logits, ids, teacher, scale, renormalise)
    loss = torch.empty(T, dtype=torch.float32, device=dev)
    stats = torch.empty((T, 2), dtype=torch.float32, device=dev)
    grad = torch.empty((T, V), dtype=logits.dtype, device=dev)
    ws, ws_at, nbytes = _workspace("bevpool_distill_workspace_size", sizes, dev)
    _call("bevpool_distill_step", *sizes, grad_loss.data_ptr(), *args, loss.data_ptr(), stats.data_ptr(),
          grad.data_ptr(), ws_at, nbytes, _stream(dev))
    return loss, grad


# ------------------------------------------------------- differentiable forms

class LogprobsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, k, scale, entropy):
        r = logprobs_forward(logits, ids, k, scale, entropy)
        ctx.scale, ctx.dtype, ctx.shape = scale, logits.dtype, logits.shape
        ctx.save_for_backward(logits, ids, r.stats, r.entropy, r.top_ids)
        ctx.mark_non_differentiable(r.stats, *(() if r.top_ids is None else (r.top_ids,)))
        ctx.set_materialize_grads(False)
        return r.logprob, r.lse, r.entropy, r.top, r.top_ids, r.stats

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        grads = [None if g is None else g.contiguous() for g in grads[:4]]
        if all(g is None for g in grads):
            return None, None, None, None, None
        logits, ids, stats, entropy, top_ids = ctx.saved_tensors  # (hooks may have replaced them)
        _matrix(logits, "logits", stats.device, ctx.dtype, ctx.shape)
        g_logprob, g_lse, g_entropy, g_top = grads
        return logprobs_backward(logits, Logprobs(None, None, entropy, None, top_ids, stats), ids, ctx.scale, g_logprob,
                                 g_lse, g_entropy, g_top), None, None, None, None


class DistillFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, scale, renormalise):
        loss, stats = distill_forward(logits, ids, teacher, scale, renormalise)
        ctx.args, ctx.dtype, ctx.shape = (scale, renormalise), logits.dtype, logits.shape
        ctx.save_for_backward(logits, ids, teacher, stats)
        ctx.set_materialize_grads(False)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss):
        if grad_loss is None:
            return None, None, None, None, None
        logits, ids, teacher, stats = ctx.saved_tensors  # (hooks may have replaced them)
        _matrix(logits, "logits", stats.device, ctx.dtype, ctx.shape)
        return distill_backward(grad_loss.contiguous(), logits, ids, teacher, stats, *ctx.args), None, None, None, None


def logprobs(logits: torch.Tensor, ids: torch.Tensor | None = None, k: int = 0, scale: float = 1.0,
             entropy: bool = False) -> Logprobs:
    """Differentiable logprobs_forward (in logprob, lse, entropy and top)."""
    return Logprobs(*LogprobsFunction.apply(logits, ids, k, scale, entropy))


def distill(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, scale: float = 1.0,
            renormalise: bool = True) -> torch.Tensor:
    """Differentiable distill_forward: the rows' losses (T,).  The teacher is a
    constant: one that needs a gradient is refused."""
    if teacher.requires_grad and torch.is_grad_enabled():
        raise ValueError("the teacher has no gradient here: detach it")
    return DistillFunction.apply(logits, ids, teacher, scale, renormalise)
