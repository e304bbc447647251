"""The dense operators of the block around the layer: norm, dropout, and dense products with bias, activation and
residual in their epilogue, with the gradients that training needs.  Argument marshalling only, as in layer.py, whose
conventions hold here: matrices may have strided rows, calls enqueue on `stream` and return, outputs may be given to
reuse buffers, and so may the workspace `ws` (uint8), which calls that can overlap must not share.
"""
from __future__ import annotations

import ctypes as C
import functools
from operator import index
from typing import Optional

import torch

from . import _check, _from, _ptr, lib
from .layer import _DTYPES, _float_dtype, _matrix, _queue, _whole

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def declare(L) -> None:
    """Argument types of this module's entry points."""
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.vp_layer_norm.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, C.c_float, i32, vp, i64, vp, vp]
    L.vp_layer_norm_grad_workspace.argtypes = [i64, i64]
    L.vp_layer_norm_grad_workspace.restype = sz
    L.vp_layer_norm_grad.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, vp, i32, i32, vp, i64, vp, i64, vp, vp, vp, sz, vp]
    L.vp_dropout.argtypes = [vp, i32, i64, i64, i64, C.c_double, C.c_uint64, vp, vp, i64, vp, i64, vp]
    L.vp_linear_workspace.argtypes = [i32, i64, i32, i32]
    L.vp_linear_workspace.restype = sz
    L.vp_linear_kernel.argtypes = [i32, i64, i32, i32, C.POINTER(i32)]
    L.vp_linear.argtypes = [vp, i64, i32, vp, i64, i64, i32, i32, vp, i32, i32, vp, i64, vp, i32, i64, vp, i64, vp, sz, vp]
    L.vp_linear_act_grad_workspace.argtypes = [i64, i64]
    L.vp_linear_act_grad_workspace.restype = sz
    L.vp_linear_act_grad.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i64, vp, vp, sz, vp]
    L.vp_linear_grad_x.argtypes = [vp, i64, i32, vp, i64, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, sz, vp]
    L.vp_linear_grad_w.argtypes = [vp, i64, vp, i64, i32, i64, i32, i32, vp, vp, sz, vp]


def _vector(t: Optional[torch.Tensor], n: int, dtype, name: str) -> int:
    """Checks a parameter vector, fp32 or of the rows' type; its type's code (fp32's where there is none)."""
    if t is None:
        return 0
    if t.dtype != torch.float32 and t.dtype != dtype:
        raise ValueError("%s must be fp32 or %s" % (name, dtype))
    _whole(t, t.dtype, (n,), name)
    return _DTYPES[t.dtype]


def _workspace(ws: Optional[torch.Tensor], need: int, device, stream) -> Optional[torch.Tensor]:
    if ws is None:
        return _from(stream, torch.empty, need, dtype=torch.uint8, device=device) if need else None
    if not ws.is_cuda or ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.numel() < need:
        raise ValueError("ws must be at least %d contiguous bytes (uint8) on the GPU" % need)
    return ws


def _act(act: str) -> int:
    if act not in ACTS:
        raise ValueError("act must be one of %s" % sorted(ACTS))
    return ACTS[act]


# ------------------------------------------------------------------ norm

def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5, center: bool = True, out: Optional[torch.Tensor] = None,
               stats: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_layer_norm over the rows of x [T, H] (fp32, bf16 or fp16), weight and bias [H] both fp32 or both of x's type;
    center=False is the root mean square's norm.  stats, fp32 [T, 2], takes what the gradient needs.  out may be x."""
    ld, dt = _matrix(x, "x"), _float_dtype(x, "x")
    T, H = x.shape
    pw, pb = _vector(weight, H, x.dtype, "weight"), _vector(bias, H, x.dtype, "bias")
    if weight is not None and bias is not None and pw != pb:
        raise ValueError("weight and bias must be of one type")
    if out is None:
        out = _from(stream, torch.empty, (T, H), dtype=x.dtype, device=x.device)
    ldo = _matrix(out, "out", cols=H, dtype=x.dtype, rows=T)
    if stats is not None:
        _whole(stats, torch.float32, (T, 2), "stats")
    queue = _queue(stream, x, weight, bias, out, stats)
    size = x.element_size()
    _check(lib().vp_layer_norm(_ptr(x), dt, T, H, ld * size, _ptr(weight), _ptr(bias), pb if weight is None else pw, eps,
                               int(center), _ptr(out), ldo * size, _ptr(stats), queue), "vp_layer_norm")
    return out


def layer_norm_grad_workspace_bytes(T: int, H: int) -> int:
    return int(lib().vp_layer_norm_grad_workspace(T, H))


def layer_norm_grad(d_out: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, weight: Optional[torch.Tensor] = None, *,
                    center: bool = True, residual: Optional[torch.Tensor] = None, params: bool = True,
                    d_x: Optional[torch.Tensor] = None, d_weight: Optional[torch.Tensor] = None,
                    d_bias: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """vp_layer_norm_grad: (d_x [T, H], d_weight, d_bias fp32 [H]); d_x has `residual` added, the gradient that reached x
    by another way.  params=False leaves the last two out (None).  d_x may be d_out or residual."""
    ldx, dt = _matrix(x, "x"), _float_dtype(x, "x")
    T, H = x.shape
    ldd = _matrix(d_out, "d_out", cols=H, dtype=x.dtype, rows=T)
    _whole(stats, torch.float32, (T, 2), "stats")
    pw = _vector(weight, H, x.dtype, "weight")
    ldr = 0 if residual is None else _matrix(residual, "residual", cols=H, dtype=x.dtype, rows=T)
    if d_x is None:
        d_x = _from(stream, torch.empty, (T, H), dtype=x.dtype, device=x.device)
    ldo = _matrix(d_x, "d_x", cols=H, dtype=x.dtype, rows=T)
    if params:
        if d_weight is None:
            d_weight = _from(stream, torch.empty, H, dtype=torch.float32, device=x.device)
        if d_bias is None:
            d_bias = _from(stream, torch.empty, H, dtype=torch.float32, device=x.device)
        _whole(d_weight, torch.float32, (H,), "d_weight")
        _whole(d_bias, torch.float32, (H,), "d_bias")
        ws = _workspace(ws, layer_norm_grad_workspace_bytes(T, H), x.device, stream)
    elif d_weight is not None or d_bias is not None:
        raise ValueError("d_weight and d_bias are not written with params=False")
    queue = _queue(stream, x, d_out, stats, weight, residual, d_x, d_weight, d_bias, ws)
    size = x.element_size()
    _check(lib().vp_layer_norm_grad(_ptr(d_out), ldd * size, _ptr(x), ldx * size, dt, T, H, _ptr(stats), _ptr(weight), pw,
                                    int(center), _ptr(residual), ldr * size, _ptr(d_x), ldo * size, _ptr(d_weight),
                                    _ptr(d_bias), _ptr(ws), 0 if ws is None else ws.numel(), queue), "vp_layer_norm_grad")
    return d_x, d_weight, d_bias


# --------------------------------------------------------------- dropout

def dropout(x: torch.Tensor, p: float, seed: int, *, step: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_dropout: x [T, H] with values dropped at probability p and the others scaled, plus residual.  The mask follows
    from seed (64 bits) and step (int64 [1] on the GPU; a captured graph that counts it up gets a new mask each replay);
    the gradient is dropout(d_out, p, seed, step=step) with the same values.  out may be x or residual."""
    ld, dt = _matrix(x, "x"), _float_dtype(x, "x")
    T, H = x.shape
    seed = index(seed)
    if not 0 <= seed < 1 << 64:
        raise ValueError("seed must be of 64 bits and not negative")   # ctypes would keep the low bits
    if step is not None:
        _whole(step, torch.int64, (1,), "step")
    ldr = 0 if residual is None else _matrix(residual, "residual", cols=H, dtype=x.dtype, rows=T)
    if out is None:
        out = _from(stream, torch.empty, (T, H), dtype=x.dtype, device=x.device)
    ldo = _matrix(out, "out", cols=H, dtype=x.dtype, rows=T)
    queue = _queue(stream, x, step, residual, out)
    size = x.element_size()
    _check(lib().vp_dropout(_ptr(x), dt, T, H, ld * size, p, seed, _ptr(step), _ptr(residual), ldr * size, _ptr(out),
                            ldo * size, queue), "vp_dropout")
    return out


# -------------------------------------------------------- dense products

def _weights2(w: torch.Tensor, dtype) -> int:
    return _matrix(w, "w", dtype=dtype)


_DIRECTIONS = ("forward", "grad_x", "grad_w")


def _fits(R: int, N: int, K: int) -> bool:
    return abs(R) < 1 << 63 and max(abs(N), abs(K)) < 1 << 31   # ctypes would keep the low bits


@functools.lru_cache(maxsize=256)
def _linear_bytes(direction: int, R: int, N: int, K: int) -> int:
    return int(lib().vp_linear_workspace(direction, R, N, K)) if _fits(R, N, K) else 0


def linear_workspace_bytes(R: int, N: int, K: int, direction: str = "forward") -> int:
    """vp_linear_workspace; direction "forward", "grad_x" or "grad_w"."""
    return _linear_bytes(_DIRECTIONS.index(direction), R, N, K)


def linear_kernel(R: int, N: int, K: int, direction: str = "forward"):
    """vp_linear_kernel: ("few_rows", "tiles_128", "tiles_256" or "tiles_alone", parts of the contraction), by which a
    product of these sizes is computed."""
    parts = C.c_int32()
    kind = lib().vp_linear_kernel(_DIRECTIONS.index(direction), R, N, K, C.byref(parts)) if _fits(R, N, K) else -1
    if kind < 0:
        raise ValueError("no product has these sizes")
    return ("few_rows", "tiles_128", "tiles_256", "tiles_alone")[kind], parts.value


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *, act: str = "none",
           residual: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
           out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """vp_linear: act(x w^T + bias) + residual [R, N] for x [R, K], w [N, K] bf16 or fp16; act of "none", "relu", "silu",
    "gelu" and "gelu_tanh".  The result, and residual with it, is of x's type or fp32 (`dtype`); `pre` of x's type takes
    x w^T + bias.  out may be residual."""
    dt = _float_dtype(x, "x", halves=True)
    ldw = _weights2(w, x.dtype)
    N, K = w.shape
    ldx = _matrix(x, "x", cols=K)
    R = x.shape[0]
    pb = _vector(bias, N, x.dtype, "bias")
    if out is None:
        out = _from(stream, torch.empty, (R, N), dtype=dtype or x.dtype, device=x.device)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError("out must be %s" % dtype)
    ldo, do, size = _matrix(out, "out", cols=N, rows=R), _float_dtype(out, "out"), out.element_size()
    ldr = 0 if residual is None else _matrix(residual, "residual", cols=N, dtype=out.dtype, rows=R)
    ldp = 0 if pre is None else _matrix(pre, "pre", cols=N, dtype=x.dtype, rows=R)
    ws = _workspace(ws, _linear_bytes(0, R, N, K), x.device, stream)
    queue = _queue(stream, x, w, bias, residual, out, pre, ws)
    _check(lib().vp_linear(_ptr(x), 2 * ldx, dt, _ptr(w), 2 * ldw, R, N, K, _ptr(bias), pb, _act(act), _ptr(residual),
                           size * ldr, _ptr(out), do, size * ldo, _ptr(pre), 2 * ldp, _ptr(ws),
                           0 if ws is None else ws.numel(), queue), "vp_linear")
    return out


def linear_act_grad_workspace_bytes(R: int, N: int) -> int:
    return int(lib().vp_linear_act_grad_workspace(R, N))


def linear_act_grad(d_y: torch.Tensor, pre: Optional[torch.Tensor] = None, *, act: str = "none", bias: bool = True,
                    out: Optional[torch.Tensor] = None, d_bias: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, stream=None):
    """vp_linear_act_grad: (d_pre [R, N], d_bias fp32 [N]) from d_y and the `pre` that linear() left; without an
    activation d_pre is d_y itself, unless `out` is given.  bias=False leaves d_bias out (None).  out may be d_y."""
    ldd, dt = _matrix(d_y, "d_y"), _float_dtype(d_y, "d_y")
    R, N = d_y.shape
    code = _act(act)
    ldp = 0 if pre is None else _matrix(pre, "pre", cols=N, dtype=d_y.dtype, rows=R)
    if (code == 0) != (pre is None):
        raise ValueError("an activation's gradient needs pre, and only that does")
    if out is None and code != 0:
        out = _from(stream, torch.empty, (R, N), dtype=d_y.dtype, device=d_y.device)
    ldo = 0 if out is None else _matrix(out, "out", cols=N, dtype=d_y.dtype, rows=R)
    if bias:
        if d_bias is None:
            d_bias = _from(stream, torch.empty, N, dtype=torch.float32, device=d_y.device)
        _whole(d_bias, torch.float32, (N,), "d_bias")
        ws = _workspace(ws, linear_act_grad_workspace_bytes(R, N), d_y.device, stream)
    elif d_bias is not None:
        raise ValueError("d_bias is not written with bias=False")
    queue = _queue(stream, d_y, pre, out, d_bias, ws)
    size = d_y.element_size()
    if out is not None or bias:
        _check(lib().vp_linear_act_grad(_ptr(d_y), ldd * size, _ptr(pre), ldp * size, dt, R, N, code, _ptr(out),
                                        ldo * size, _ptr(d_bias), _ptr(ws), 0 if ws is None else ws.numel(), queue),
               "vp_linear_act_grad")
    return (d_y if out is None else out), d_bias


def linear_grad_x(d_y: torch.Tensor, w: torch.Tensor, *, act: str = "none", pre: Optional[torch.Tensor] = None,
                  residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_linear_grad_x: (d_y w) * act'(pre) + residual [R, K]: with the act and pre of the product that made x, the
    gradient goes on through that activation.  out may be residual."""
    dt = _float_dtype(d_y, "d_y", halves=True)
    ldw = _weights2(w, d_y.dtype)
    N, K = w.shape
    ldd = _matrix(d_y, "d_y", cols=N)
    R = d_y.shape[0]
    code = _act(act)
    if (code == 0) != (pre is None):
        raise ValueError("an activation's gradient needs pre, and only that does")
    ldp = 0 if pre is None else _matrix(pre, "pre", cols=K, dtype=d_y.dtype, rows=R)
    ldr = 0 if residual is None else _matrix(residual, "residual", cols=K, dtype=d_y.dtype, rows=R)
    if out is None:
        out = _from(stream, torch.empty, (R, K), dtype=d_y.dtype, device=d_y.device)
    ldo = _matrix(out, "out", cols=K, dtype=d_y.dtype, rows=R)
    ws = _workspace(ws, _linear_bytes(1, R, N, K), d_y.device, stream)
    queue = _queue(stream, d_y, w, pre, residual, out, ws)
    _check(lib().vp_linear_grad_x(_ptr(d_y), 2 * ldd, dt, _ptr(w), 2 * ldw, R, N, K, code, _ptr(pre), 2 * ldp,
                                  _ptr(residual), 2 * ldr, _ptr(out), 2 * ldo, _ptr(ws), 0 if ws is None else ws.numel(),
                                  queue), "vp_linear_grad_x")
    return out


def linear_grad_w(d_y: torch.Tensor, x: torch.Tensor, *, out: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_linear_grad_w: d_y^T x, fp32 [N, K]."""
    dt = _float_dtype(d_y, "d_y", halves=True)
    ldd = _matrix(d_y, "d_y")
    R, N = d_y.shape
    ldx = _matrix(x, "x", dtype=d_y.dtype, rows=R)
    K = x.shape[1]
    if out is None:
        out = _from(stream, torch.empty, (N, K), dtype=torch.float32, device=d_y.device)
    _whole(out, torch.float32, (N, K), "out")
    ws = _workspace(ws, _linear_bytes(2, R, N, K), d_y.device, stream)
    queue = _queue(stream, d_y, x, out, ws)
    _check(lib().vp_linear_grad_w(_ptr(d_y), 2 * ldd, _ptr(x), 2 * ldx, dt, R, N, K, _ptr(out), _ptr(ws),
                                  0 if ws is None else ws.numel(), queue), "vp_linear_grad_w")
    return out
