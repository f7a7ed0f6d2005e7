"""Row operators of libbevpool.so (include/bevpool_rows.h): router, dispatch
and combine of expert layers, embedding lookup, and the stable key sort they
share.

They are the moves of the pooling path for keys that are expert ids or row
ids: ``sort_keys`` orders slots by key as ``prepare`` orders frustum points by
cell, and rows are read through that order and summed without atomics.  Keys
outside their range (padding, a token past an expert's capacity) are dropped:
they sort last, their rows are zero and carry no gradient.

``*_forward`` and ``*_backward`` allocate their outputs and launch the kernels;
``route``, ``dispatch``, ``combine`` and ``embed`` are their differentiable
forms.  A layer of experts reads

    weights, ids = route(logits, k)
    rows, plan = dispatch(x, ids, n_experts)      # rows of expert e:
    y = experts(rows, plan.offsets)               #   offsets[e] .. offsets[e+1]
    out = combine(y, weights, plan)

Matrices may have any distance between their rows (a slice of a wider matrix,
one row expanded); elements of a row are neighbours.  Everything runs on the
tensors' device and its current stream, or on ``stream``, which the inputs then
have to be ready on.  No call synchronises or reads back.

Into a HIP graph the ``*_forward`` and ``*_backward`` calls are captured as they
are.  A backward pass through the differentiable forms is captured under torch's
own rule: no graph of the same leaves made outside the capture may be alive, or
their gradients are added up on a stream that does not take part in it.

A differentiable form keeps for its gradient only what that reads: the router's
logits where its weights are not renormalised, the rows of a combine where its
weights need a gradient, the weights where the rows do.
"""

from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import bevpool as _bp

BEVPOOL_BF16 = 2
BEVPOOL_KEY_I32, BEVPOOL_KEY_I64 = 0, 1

_DTYPE_CODE = {torch.float32: _bp.BEVPOOL_F32, torch.float16: _bp.BEVPOOL_F16, torch.bfloat16: BEVPOOL_BF16}
_KEY_CODE = {torch.int32: BEVPOOL_KEY_I32, torch.int64: BEVPOOL_KEY_I64}
_I32, _F32 = (torch.int32,), (torch.float32,)

_vp, _i32, _i64, _int, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
_ARGTYPES = {
    "bevpool_sort_keys_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "bevpool_sort_keys": [_i64, _i64, _int, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "bevpool_route_forward": [_i64, _i32, _i32, _int, _vp, _i64, _int, _vp, _vp, _vp],
    "bevpool_route_backward": [_i64, _i32, _i32, _int, _vp, _vp, _i64, _vp, _vp, _int, _vp, _vp],
    "bevpool_dispatch_forward": [_i64, _i32, _i64, _i64, _int, _vp, _i64, _int, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                 _vp],
    "bevpool_dispatch_rows": [_i64, _i32, _i64, _int, _vp, _i64, _vp, _vp, _vp, _vp],
    "bevpool_dispatch_backward": [_i64, _i32, _i64, _int, _vp, _i64, _vp, _vp, _vp, _vp],
    "bevpool_combine_forward": [_i64, _i32, _i64, _int, _int, _int, _vp, _i64, _vp, _vp, _vp, _vp, _vp],
    "bevpool_combine_backward": [_i64, _i32, _i64, _int, _int, _int, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp,
                                 _vp],
    "bevpool_embed_forward": [_i64, _i64, _i64, _int, _int, _vp, _i64, _int, _vp, ctypes.c_float, _vp, _vp],
    "bevpool_embed_backward_workspace_size": [_i64, _i64, _i64, ctypes.POINTER(_sz)],
    "bevpool_embed_backward": [_i64, _i64, _i64, _int, _int, _vp, _i64, _int, _vp, ctypes.c_float, _vp, _vp, _sz,
                               _vp],
}

_lib = None


def load_library() -> ctypes.CDLL:
    """libbevpool.so with the row operators' signatures (raises if it has not been built)."""
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


@functools.lru_cache(maxsize=1024)
def _size(name: str, *args) -> int:
    n = _sz(0)
    _call(name, *args, ctypes.byref(n))
    return n.value


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(dev: torch.device) -> int:
    """Handle of dev's current stream (torch's raw query costs a tenth of a stream object)."""
    return _bp._raw_stream(dev.index) if _bp._raw_stream else torch.cuda.current_stream(dev).cuda_stream


# ----------------------------------------------------------------- arguments

def _device(t, name: str) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    return t.device


def _matrix(t, name: str, dev: torch.device, dtype=None, shape=None) -> int:
    """Checks a matrix whose rows are runs of neighbouring elements; the
    distance between its rows."""
    if not isinstance(t, torch.Tensor) or t.device != dev:
        raise ValueError(f"{name} must be a tensor on {dev}")
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be {shape or 'a matrix'}, got {tuple(t.shape)}")
    if t.dtype not in _DTYPE_CODE or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'float32, float16 or bfloat16'}, got {t.dtype}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be neighbours (stride {t.stride(1)})")
    return t.stride(0)


def _dense(t, name: str, dev: torch.device, dtypes, shape=None) -> None:
    if not isinstance(t, torch.Tensor) or t.device != dev:
        raise ValueError(f"{name} must be a tensor on {dev}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {[str(d) for d in dtypes]}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


# The library's counts of experts, of choices and of slots to a token are 32-bit
# integers, of which a larger one would pass its low bits only.
_LIMIT = 1 << 31


def _check_choices(E: int, k: int) -> None:
    if E >= _LIMIT or k >= _LIMIT:
        raise ValueError(f"{k} of {E} experts exceed 2^31 - 1")


def _elsewhere(dev: torch.device, stream, *inputs):
    """A context in which dev and `stream` are current, or None where they
    already are: allocations and launches then belong to that stream."""
    if stream is None:
        return None if dev.index == _current_device() else torch.cuda.device(dev)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=dev)
    if stream.device != dev:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {dev}")
    for t in inputs:  # (their memory must outlive the work on that stream)
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    return torch.cuda.stream(stream)


@dataclass
class KeyOrder:
    """Stable order of n slots by key: ``order[q]`` the slot at place q,
    ``position[s]`` the place of slot s, ``offsets[v]`` the first place of key
    v, ``offsets[n_keys]`` the number of kept slots (dropped ones lie behind).
    ``k``: the slots of a token, where a dispatch made the order.  The moves go
    by position and offsets: ``order`` may be None."""
    order: torch.Tensor | None
    position: torch.Tensor
    offsets: torch.Tensor
    n_keys: int
    k: int | None = None

    def _check(self, dev: torch.device, n: int, k: int) -> int:
        """Address of the number of kept slots, of n slots, k to a token."""
        position, offsets, n_keys = self.position, self.offsets, self.n_keys
        _dense(position, "position", dev, _I32)
        _dense(offsets, "offsets", dev, _I32)
        if not position.numel() == n < _LIMIT or not offsets.numel() == n_keys + 1 > 0:
            if n >= _LIMIT:
                raise ValueError(f"{n} slots exceed 2^31 - 1")
            if n_keys < 0:  # (the count would lie before the offsets)
                raise ValueError(f"n_keys = {n_keys} is negative")
            raise ValueError(f"the order has {position.numel()} slots and {offsets.numel()} offsets; "
                             f"{n} slots and {n_keys + 1} offsets are needed")
        if self.k is not None and self.k != k and n > 0:
            raise ValueError(f"the order has {self.k} slots to a token, not {k}")
        return offsets.data_ptr() + 4 * n_keys


def _key_order(keys: torch.Tensor, n_keys: int, dev: torch.device, k: int | None = None):
    n = keys.numel()
    nbytes = _size("bevpool_sort_keys_workspace_size", n, n_keys)
    i32 = torch.int32
    plan = KeyOrder(torch.empty(n, dtype=i32, device=dev), torch.empty(n, dtype=i32, device=dev),
                    torch.empty(n_keys + 1, dtype=i32, device=dev), n_keys, k)
    return plan, torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None, nbytes


# --------------------------------------------------------------- key sorting

def sort_keys(keys: torch.Tensor, n_keys: int, stream=None) -> KeyOrder:
    """Stable order of integer keys (any shape, int32 or int64) in [0, n_keys);
    keys outside are dropped.  A key is a slot; how many of them make a token is
    the caller's to say, by the rows that go through the order."""
    dev = _device(keys, "keys")
    _dense(keys, "keys", dev, _KEY_CODE)
    ctx = _elsewhere(dev, stream, keys)
    if ctx is not None:
        with ctx:
            return sort_keys(keys, n_keys)
    plan, ws, nbytes = _key_order(keys, n_keys, dev)
    _call("bevpool_sort_keys", keys.numel(), n_keys, _KEY_CODE[keys.dtype], keys.data_ptr(), plan.order.data_ptr(),
          plan.position.data_ptr(), plan.offsets.data_ptr(), _bp._ptr(ws), nbytes, _stream(dev))
    return plan


# -------------------------------------------------------------------- router

def route_forward(logits: torch.Tensor, k: int, renormalise: bool = True, stream=None):
    """(weights, ids) of the k largest logits (T, E) of every row: ids (T, k)
    int32 by descending logit, equal logits by index, -1 where fewer than k are
    above -inf; weights (T, k) float32, their softmax over the chosen
    (renormalise) or over all experts."""
    dev = _device(logits, "logits")
    stride = _matrix(logits, "logits", dev)
    T, E = logits.shape
    _check_choices(E, k)
    ctx = _elsewhere(dev, stream, logits)
    if ctx is not None:
        with ctx:
            return route_forward(logits, k, renormalise)
    weights = torch.empty((T, k), dtype=torch.float32, device=dev)
    ids = torch.empty((T, k), dtype=torch.int32, device=dev)
    _call("bevpool_route_forward", T, E, k, _DTYPE_CODE[logits.dtype], logits.data_ptr(), stride, int(renormalise),
          weights.data_ptr(), ids.data_ptr(), _stream(dev))
    return weights, ids


def route_backward(grad_weights: torch.Tensor, logits: torch.Tensor, weights: torch.Tensor, ids: torch.Tensor,
                   renormalise: bool = True, stream=None) -> torch.Tensor:
    """Gradient (T, E) of the logits, in their type."""
    dev = _device(logits, "logits")
    _matrix(logits, "logits", dev)
    T, E = logits.shape
    k = ids.shape[-1]
    _check_choices(E, k)
    _dense(grad_weights, "grad_weights", dev, _F32, (T, k))
    _dense(weights, "weights", dev, _F32, (T, k))
    _dense(ids, "ids", dev, _I32, (T, k))
    ctx = _elsewhere(dev, stream, grad_weights, logits, weights, ids)
    if ctx is not None:
        with ctx:
            return route_backward(grad_weights, logits, weights, ids, renormalise)
    return _route_gradient(grad_weights, None if renormalise else logits, weights, ids, E, logits.dtype)


def _route_gradient(grad_weights, logits, weights, ids, E: int, dtype: torch.dtype) -> torch.Tensor:
    """route_backward without its checks; logits None: of renormalised weights, whose gradient does not read them."""
    dev = ids.device
    T, k = ids.shape
    grad = torch.empty((T, E), dtype=dtype, device=dev)
    _call("bevpool_route_backward", T, E, k, _DTYPE_CODE[dtype], grad_weights.data_ptr(), _bp._ptr(logits),
          0 if logits is None else logits.stride(0), weights.data_ptr(), ids.data_ptr(), int(logits is None),
          grad.data_ptr(), _stream(dev))
    return grad


# ------------------------------------------------------- dispatch and combine

def dispatch_forward(x: torch.Tensor, ids, n_experts: int | None = None, stream=None):
    """(rows, plan): the rows of x (T, C) in the order of their experts, one for
    every slot of ids (T, k), and that order.  Rows of dropped slots lie behind
    the kept ones and are zero.  ``ids`` may also be the KeyOrder of an earlier
    call with T rows."""
    dev = _device(x, "x")
    stride = _matrix(x, "x", dev)
    T, C = x.shape
    if isinstance(ids, KeyOrder):
        plan = ids
        n = plan.position.numel()
        k = n // T if T else 1
        kept = plan._check(dev, T * k, k)
    else:
        _dense(ids, "ids", dev, _KEY_CODE)
        if ids.dim() != 2 or ids.shape[0] != T:
            raise ValueError(f"ids must be ({T}, k), got {tuple(ids.shape)}")
        if n_experts is None:
            raise ValueError("n_experts is needed with ids")
        plan = None
        k, n = ids.shape[1], ids.numel()
    ctx = _elsewhere(dev, stream, x, *((ids,) if plan is None else (plan.position, plan.offsets)))
    if ctx is not None:
        with ctx:
            return dispatch_forward(x, ids, n_experts)
    out = torch.empty((n, C), dtype=x.dtype, device=dev)
    if plan is not None:
        _call("bevpool_dispatch_rows", T, k, C, _DTYPE_CODE[x.dtype], x.data_ptr(), stride, plan.position.data_ptr(),
              kept, out.data_ptr(), _stream(dev))
        return out, plan
    plan, ws, nbytes = _key_order(ids, n_experts, dev, k)
    _call("bevpool_dispatch_forward", T, k, C, n_experts, _DTYPE_CODE[x.dtype], x.data_ptr(), stride,
          _KEY_CODE[ids.dtype], ids.data_ptr(), plan.order.data_ptr(), plan.position.data_ptr(),
          plan.offsets.data_ptr(), out.data_ptr(), _bp._ptr(ws), nbytes, _stream(dev))
    return out, plan


def _tokens(rows: torch.Tensor, k: int) -> int:
    if k < 1 or rows.shape[0] % k:
        raise ValueError(f"{rows.shape[0]} rows are not a multiple of k = {k}")
    return rows.shape[0] // k


def dispatch_backward(grad_rows: torch.Tensor, plan: KeyOrder, k: int, stream=None) -> torch.Tensor:
    """Gradient (T, C) of x from that of the dispatched rows (T k, C)."""
    dev = _device(grad_rows, "grad_rows")
    stride = _matrix(grad_rows, "grad_rows", dev)
    T = _tokens(grad_rows, k)
    kept = plan._check(dev, T * k, k)
    ctx = _elsewhere(dev, stream, grad_rows, plan.position, plan.offsets)
    if ctx is not None:
        with ctx:
            return dispatch_backward(grad_rows, plan, k)
    C = grad_rows.shape[1]
    grad = torch.empty((T, C), dtype=grad_rows.dtype, device=dev)
    _call("bevpool_dispatch_backward", T, k, C, _DTYPE_CODE[grad_rows.dtype], grad_rows.data_ptr(), stride,
          plan.position.data_ptr(), kept, grad.data_ptr(), _stream(dev))
    return grad


def combine_forward(rows: torch.Tensor, weights: torch.Tensor, plan: KeyOrder, out_dtype=None,
                    stream=None) -> torch.Tensor:
    """(T, C): the sum of every token's kept rows, out of rows (T k, C) in the
    order of their experts, times its weights (T, k; float32 or rows' type).
    out_dtype: rows' type (default) or float32."""
    dev = _device(rows, "rows")
    stride = _matrix(rows, "rows", dev)
    _dense(weights, "weights", dev, (torch.float32, rows.dtype))
    n, C = rows.shape
    if weights.dim() != 2 or weights.numel() != n:
        raise ValueError(f"weights must be (T, k) for {n} rows, got {tuple(weights.shape)}")
    T, k = weights.shape
    kept = plan._check(dev, n, k)
    odt = out_dtype or rows.dtype
    if odt not in (rows.dtype, torch.float32):
        raise ValueError(f"out_dtype must be {rows.dtype} or float32, got {odt}")
    ctx = _elsewhere(dev, stream, rows, weights, plan.position, plan.offsets)
    if ctx is not None:
        with ctx:
            return combine_forward(rows, weights, plan, out_dtype)
    out = torch.empty((T, C), dtype=odt, device=dev)
    _call("bevpool_combine_forward", T, k, C, _DTYPE_CODE[rows.dtype], _DTYPE_CODE[odt], _DTYPE_CODE[weights.dtype],
          rows.data_ptr(), stride, weights.data_ptr(), plan.position.data_ptr(), kept, out.data_ptr(),
          _stream(dev))
    return out


def combine_backward(grad_out: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor, plan: KeyOrder,
                     need_rows: bool = True, need_weights: bool = True, stream=None):
    """(grad_rows, grad_weights) of combine_forward, in the types of rows and
    weights; None for one that is not needed."""
    dev = _device(rows, "rows")
    stride = _matrix(rows, "rows", dev)
    _dense(weights, "weights", dev, (torch.float32, rows.dtype))
    n, C = rows.shape
    if weights.dim() != 2 or weights.numel() != n:
        raise ValueError(f"weights must be (T, k) for {n} rows, got {tuple(weights.shape)}")
    T, k = weights.shape
    grad_stride = _matrix(grad_out, "grad_out", dev, shape=(T, C))
    if grad_out.dtype not in (rows.dtype, torch.float32):
        raise ValueError(f"grad_out must be {rows.dtype} or float32, got {grad_out.dtype}")
    kept = plan._check(dev, n, k)
    ctx = _elsewhere(dev, stream, grad_out, rows, weights, plan.position, plan.offsets)
    if ctx is not None:
        with ctx:
            return combine_backward(grad_out, rows, weights, plan, need_rows, need_weights)
    return _combine_gradients(grad_out, grad_stride, rows if need_weights else None, stride,
                              weights if need_rows else None, plan.position, kept, (T, k, C), rows.dtype,
                              weights.dtype)


def _combine_gradients(grad_out, grad_stride: int, rows, stride: int, weights, position, kept: int, shape, rows_dtype,
                       weights_dtype):
    """combine_backward without its checks (kept: the address of the count): the gradient of the rows where the
    weights are given, that of the weights where the rows are (each reads the other operand only)."""
    dev = grad_out.device
    T, k, C = shape
    grad_rows = rows_at = weights_at = grad_rows_at = grad_weights = grad_weights_at = None
    if weights is not None:
        grad_rows = torch.empty((T * k, C), dtype=rows_dtype, device=dev)
        weights_at, grad_rows_at = weights.data_ptr(), grad_rows.data_ptr()
    if rows is not None:
        grad_weights = torch.empty((T, k), dtype=weights_dtype, device=dev)
        rows_at, grad_weights_at = rows.data_ptr(), grad_weights.data_ptr()
    _call("bevpool_combine_backward", T, k, C, _DTYPE_CODE[rows_dtype], _DTYPE_CODE[grad_out.dtype],
          _DTYPE_CODE[weights_dtype], grad_out.data_ptr(), grad_stride, rows_at, stride, weights_at,
          position.data_ptr(), kept, grad_rows_at, grad_weights_at, _stream(dev))
    return grad_rows, grad_weights


# ----------------------------------------------------------------- embedding

def embed_forward(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype=None,
                  stream=None) -> torch.Tensor:
    """scale * table[ids] of shape ids.shape + (C,); zeros for ids outside the
    table.  out_dtype: the table's type (default) or float32."""
    dev = _device(table, "table")
    stride = _matrix(table, "table", dev)
    _dense(ids, "ids", dev, _KEY_CODE)
    odt = out_dtype or table.dtype
    if odt not in (table.dtype, torch.float32):
        raise ValueError(f"out_dtype must be {table.dtype} or float32, got {odt}")
    ctx = _elsewhere(dev, stream, table, ids)
    if ctx is not None:
        with ctx:
            return embed_forward(table, ids, scale, out_dtype)
    V, C = table.shape
    out = torch.empty(ids.shape + (C,), dtype=odt, device=dev)
    _call("bevpool_embed_forward", ids.numel(), V, C, _DTYPE_CODE[table.dtype], _DTYPE_CODE[odt], table.data_ptr(),
          stride, _KEY_CODE[ids.dtype], ids.data_ptr(), scale, out.data_ptr(), _stream(dev))
    return out


def embed_backward(grad_out: torch.Tensor, ids: torch.Tensor, table_rows: int, scale: float = 1.0, grad_dtype=None,
                   stream=None) -> torch.Tensor:
    """Gradient (table_rows, C) of the table, zeros in rows that no id names.
    grad_dtype: grad_out's type (default), float32, or any type when grad_out
    is float32."""
    dev = _device(ids, "ids")
    _dense(ids, "ids", dev, _KEY_CODE)
    if not isinstance(grad_out, torch.Tensor) or grad_out.dim() < 1 or grad_out.shape[:-1] != ids.shape:
        raise ValueError(f"grad_out must be {tuple(ids.shape)} + (C,)")
    if grad_out.dim() != 2:
        if not grad_out.is_contiguous():
            raise ValueError("grad_out must be contiguous or a matrix")
        grad_out = grad_out.view(ids.numel(), grad_out.shape[-1])
    stride = _matrix(grad_out, "grad_out", dev)
    gdt = grad_dtype or grad_out.dtype
    if gdt not in _DTYPE_CODE or (gdt != grad_out.dtype and torch.float32 not in (gdt, grad_out.dtype)):
        raise ValueError(f"grad_dtype {gdt} does not go with a grad_out of {grad_out.dtype}")
    ctx = _elsewhere(dev, stream, grad_out, ids)
    if ctx is not None:
        with ctx:
            return embed_backward(grad_out.view(ids.shape + grad_out.shape[-1:]) if ids.dim() != 1 else grad_out, ids,
                                  table_rows, scale, grad_dtype)
    n, C = grad_out.shape
    grad = torch.empty((table_rows, C), dtype=gdt, device=dev)
    nbytes = _size("bevpool_embed_backward_workspace_size", n, table_rows, C)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _call("bevpool_embed_backward", n, table_rows, C, _DTYPE_CODE[grad_out.dtype], _DTYPE_CODE[gdt],
          grad_out.data_ptr(), stride, _KEY_CODE[ids.dtype], ids.data_ptr(), scale, grad.data_ptr(), ws.data_ptr(),
          nbytes, _stream(dev))
    return grad


# ------------------------------------------------------- differentiable forms

class RouteFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, renormalise):
        weights, ids = route_forward(logits, k, renormalise)
        ctx.experts, ctx.dtype = logits.shape[1], logits.dtype
        ctx.save_for_backward(None if renormalise else logits, weights, ids)
        ctx.mark_non_differentiable(ids)
        ctx.set_materialize_grads(False)
        return weights, ids

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_weights, _):
        if grad_weights is None:
            return None, None, None
        logits, weights, ids = ctx.saved_tensors  # (hooks may have replaced them)
        dev, shape = grad_weights.device, grad_weights.shape
        _dense(weights, "weights", dev, _F32, shape)
        _dense(ids, "ids", dev, _I32, shape)
        if logits is not None:
            _matrix(logits, "logits", dev, ctx.dtype, (shape[0], ctx.experts))
        return _route_gradient(grad_weights.contiguous(), logits, weights, ids, ctx.experts, ctx.dtype), None, None


class DispatchFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, ids, n_experts):
        rows, plan = dispatch_forward(x, ids, n_experts)
        ctx.n_keys, ctx.tokens = plan.n_keys, x.shape[0]
        ctx.save_for_backward(plan.position, plan.offsets)
        ctx.set_materialize_grads(False)
        if isinstance(ids, KeyOrder):
            return rows
        ctx.mark_non_differentiable(plan.order, plan.position, plan.offsets)
        return rows, plan.order, plan.position, plan.offsets

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_rows, *_):
        if grad_rows is None:
            return None, None, None
        position, offsets = ctx.saved_tensors
        plan = KeyOrder(None, position, offsets, ctx.n_keys)
        k = position.numel() // ctx.tokens if ctx.tokens else 1
        return dispatch_backward(_rows_apart(grad_rows), plan, k), None, None


class CombineFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, weights, plan, out_dtype):
        out = combine_forward(rows, weights, plan, out_dtype)
        need_rows, need_weights = ctx.needs_input_grad[:2]
        ctx.n_keys, ctx.shape, ctx.dtypes = plan.n_keys, (*weights.shape, rows.shape[1]), (rows.dtype, weights.dtype)
        ctx.save_for_backward(rows if need_weights else None, weights if need_rows else None, plan.position,
                              plan.offsets)
        ctx.set_materialize_grads(False)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        if grad_out is None:
            return None, None, None, None
        rows, weights, position, offsets = ctx.saved_tensors  # (hooks may have replaced them)
        need_rows, need_weights = ctx.needs_input_grad[:2]
        rows, weights = rows if need_weights else None, weights if need_rows else None
        (T, k, C), (rows_dtype, weights_dtype), dev = ctx.shape, ctx.dtypes, grad_out.device
        grad_out = _rows_apart(grad_out)
        stride = 0 if rows is None else _matrix(rows, "rows", dev, rows_dtype, (T * k, C))
        if weights is not None:
            _dense(weights, "weights", dev, (weights_dtype,), (T, k))
        kept = KeyOrder(None, position, offsets, ctx.n_keys)._check(dev, T * k, k)
        grads = _combine_gradients(grad_out, grad_out.stride(0), rows, stride, weights, position, kept, ctx.shape,
                                   rows_dtype, weights_dtype)
        return *grads, None, None


class EmbedFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, out_dtype):
        ctx.table_rows, ctx.dtype, ctx.scale = table.shape[0], table.dtype, scale
        ctx.save_for_backward(ids)
        ctx.set_materialize_grads(False)
        return embed_forward(table, ids, scale, out_dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        if grad_out is None:
            return None, None, None, None
        ids, = ctx.saved_tensors  # (hooks may have replaced them)
        grad_out = _rows_apart(grad_out) if ids.dim() == 1 else grad_out.contiguous()
        return embed_backward(grad_out, ids, ctx.table_rows, ctx.scale, ctx.dtype), None, None, None


def _rows_apart(g: torch.Tensor) -> torch.Tensor:
    """A gradient whose rows the kernels can read (a sum's gradient has stride 0 within its rows)."""
    return g if g.shape[-1] <= 1 or g.stride(-1) == 1 else g.contiguous()


def route(logits: torch.Tensor, k: int, renormalise: bool = True):
    """Differentiable route_forward: (weights, ids)."""
    return RouteFunction.apply(logits, k, renormalise)


def dispatch(x: torch.Tensor, ids, n_experts: int | None = None):
    """Differentiable dispatch_forward: (rows, plan)."""
    if isinstance(ids, KeyOrder):
        return DispatchFunction.apply(x, ids, None), ids
    rows, order, position, offsets = DispatchFunction.apply(x, ids, n_experts)
    return rows, KeyOrder(order, position, offsets, n_experts, ids.shape[1])


def combine(rows: torch.Tensor, weights: torch.Tensor, plan: KeyOrder, out_dtype=None) -> torch.Tensor:
    """Differentiable combine_forward."""
    return CombineFunction.apply(rows, weights, plan, out_dtype)


def embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype=None) -> torch.Tensor:
    """Differentiable embed_forward; the table's gradient is dense."""
    return EmbedFunction.apply(table, ids, scale, out_dtype)
