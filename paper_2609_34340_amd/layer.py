"""The layer around the exchanges: routing, the experts' products, the merge
of the returned rows and rows in 4-bit blocks, with the gradients that training
needs.  Argument marshalling only, as in the package's own module, which offers
these names too.

Matrices may have strided rows (the receive slots' 128-byte stride), their
elements must be neighbours.  Every call enqueues on `stream` (the current one
by default) and returns; outputs may be given to reuse buffers.  Errors that
only the device can see go to `status` (new_status()) where one is given, else
the first of them is kept until unclaimed_status() asks.
"""
from __future__ import annotations

import ctypes as C
import functools
from operator import index
from typing import Optional

import torch

from . import _check, _from, _ptr, _stream, lib, new_status, read_status

SCORES = {"softmax": 0, "sigmoid": 1}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MX_BLOCK = 32   # values that share one power of two


class RouteParams(C.Structure):
    _fields_ = [("score", C.c_int32), ("top_k", C.c_int32), ("n_groups", C.c_int32), ("top_groups", C.c_int32),
                ("group_top", C.c_int32), ("renorm", C.c_int32), ("scale", C.c_float)]


def declare(L) -> None:
    """Argument types of this module's entry points."""
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    route = C.POINTER(RouteParams)
    L.vp_route.argtypes = [vp, i32, i64, i32, i64, route, vp, vp, vp, vp]
    L.vp_route_grad.argtypes = [vp, i32, i64, i32, i64, route, vp, vp, vp, vp, vp, vp]
    L.vp_expert_offsets.argtypes = [vp, i32, i32, i32, vp, vp, vp]
    L.vp_expert_matmul.argtypes = [vp, i64, i32, vp, vp, i64, i32, i32, i32, i32, vp, i64, vp, i64, vp, vp]
    L.vp_expert_matmul_grad_x.argtypes = [vp, i64, i32, vp, vp, i64, i32, i32, i32, vp, i64, vp, vp]
    L.vp_expert_matmul_grad_w.argtypes = [vp, i64, vp, i64, i32, vp, i64, i32, i32, i32, vp, vp, vp]
    L.vp_expert_gate_grad.argtypes = [vp, i64, vp, i64, i32, vp, i64, i32, i32, vp, i64, vp, vp]
    L.vp_merge.argtypes = [vp, i32, i64, i32, i64, i64, vp, vp, i64, vp, i64, vp]
    L.vp_merge_grad.argtypes = [vp, i32, i64, i32, i64, i64, vp, i64, vp, vp, i64, vp, vp]
    L.vp_mx_row_bytes.argtypes = [i64]
    L.vp_mx_row_bytes.restype = i64
    L.vp_mx_quantize.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp]
    L.vp_mx_dequantize.argtypes = [vp, i64, i64, i64, vp, i32, i64, vp]
    L.vp_expert_matmul_mx.argtypes = [vp, i64, vp, vp, i64, i32, i32, i32, i32, vp, i32, i64, vp, vp]
    L.vp_take_status.argtypes = [vp, vp]
    L.vp_expert_kernel.argtypes = [i32, i32, i32, i64, i32, i32, i32]
    L.vp_route_lanes.argtypes = [i64, i32]


# The checks are written for their cost: a small call is bound by the host (a decode step's merge 10 us a pass, of which
# the kernel takes 4), and every tensor attribute is a call.

def _matrix(t: torch.Tensor, name: str, cols: Optional[int] = None, dtype=None, rows: Optional[int] = None) -> int:
    """Checks a [rows, cols] GPU matrix whose elements are neighbours; its row stride in elements."""
    shape = t.shape
    if not t.is_cuda or len(shape) != 2:
        raise ValueError("%s must be a matrix on the GPU" % name)
    n, m = shape
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s" % (name, dtype))
    if (cols is not None and m != cols) or (rows is not None and n != rows):
        raise ValueError("%s must be [%s, %s], is %s" % (name, "rows" if rows is None else rows,
                                                         "columns" if cols is None else cols, tuple(shape)))
    ld, one = t.stride()
    if one != 1 and m > 1:
        raise ValueError("%s must have neighbouring elements in a row" % name)
    if n <= 1:
        return m
    if ld < m:
        raise ValueError("%s has overlapping rows" % name)
    return ld


def _whole(t: torch.Tensor, dtype, shape, name: str) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor %s on the GPU" % (name, dtype, tuple(shape)))
    return t


def _float_dtype(t: torch.Tensor, name: str, halves: bool = False) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None or (halves and code == 0):
        raise ValueError("%s must be bf16%s" % (name, " or fp16" if halves else ", fp16 or fp32"))
    return code


def _queue(stream, first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """The handle of the stream a call runs on, once all of its tensors are known to be on that stream's device."""
    device = first.get_device()
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on one device")
    # kernels run on the current device, which need not reach another one's memory
    if device != torch.cuda.current_device() or (stream is not None and stream.device_index != device):
        raise ValueError("the tensors must be on the current device, and the stream too")
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def unclaimed_status(stream=None) -> int:
    """vp_take_status: the first device error of this module's calls that were given no status since this was last asked,
    0 if there was none.  Waits for the stream."""
    status = _from(stream, new_status)
    _check(lib().vp_take_status(_ptr(status), _stream(stream)), "vp_take_status")
    return _from(stream, read_status, status)


# --------------------------------------------------------------- routing

def _route_params(score, k, n_groups, top_groups, group_top, renorm, scale):
    """The parameter block.  Its arguments become plain values first: a tensor or array can change in place."""
    if score not in SCORES:
        raise ValueError("score must be one of %s" % sorted(SCORES))
    return _route_block(SCORES[score], index(k), index(n_groups), index(n_groups if top_groups is None else top_groups),
                        index(group_top), bool(renorm), float(scale))


@functools.lru_cache(maxsize=64)
def _route_block(score, k, n_groups, top_groups, group_top, renorm, scale):
    if max(abs(v) for v in (k, n_groups, top_groups, group_top)) >= 1 << 31:
        raise ValueError("top_k and the groups must be below 2^31")   # ctypes would keep the low bits
    return C.byref(RouteParams(score, k, n_groups, top_groups, group_top, int(renorm), scale))


def route(logits: torch.Tensor, k: int, *, score: str = "softmax", bias: Optional[torch.Tensor] = None,
          n_groups: int = 1, top_groups: Optional[int] = None, group_top: int = 1, renorm: bool = True,
          scale: float = 1.0, out: Optional[dict] = None, stream=None) -> dict:
    """vp_route over logits [T, E] (fp32, bf16 or fp16).  Returns ids int32 [T, k] (the routing that demand()
    takes, as ids[None]) and weights fp32 [T, k]."""
    ld = _matrix(logits, "logits")
    dt = _float_dtype(logits, "logits")
    T, E = logits.shape
    if bias is not None:
        _whole(bias, torch.float32, (E,), "bias")
    if out is None:
        out = dict(ids=_from(stream, torch.empty, (T, k), dtype=torch.int32, device=logits.device),
                   weights=_from(stream, torch.empty, (T, k), dtype=torch.float32, device=logits.device))
    ids = _whole(out["ids"], torch.int32, (T, k), "ids")
    weights = _whole(out["weights"], torch.float32, (T, k), "weights")
    queue = _queue(stream, logits, bias, ids, weights)
    p = _route_params(score, k, n_groups, top_groups, group_top, renorm, scale)
    _check(lib().vp_route(_ptr(logits), dt, T, E, ld, p, _ptr(bias), _ptr(ids), _ptr(weights), queue),
           "vp_route")
    return out


def route_grad(logits: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, d_weights: torch.Tensor, *,
               score: str = "softmax", renorm: bool = True, scale: float = 1.0, out: Optional[torch.Tensor] = None,
               status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_route_grad: d_logits [T, E] of the logits' type from d_weights and what route() returned."""
    ld = _matrix(logits, "logits")
    dt = _float_dtype(logits, "logits")
    T, E = logits.shape
    if ids.dim() != 2:
        raise ValueError("ids must be [T, k]")
    k = ids.shape[1]
    _whole(ids, torch.int32, (T, k), "ids")
    _whole(weights, torch.float32, (T, k), "weights")
    _whole(d_weights, torch.float32, (T, k), "d_weights")
    if out is None:
        out = _from(stream, torch.empty, (T, E), dtype=logits.dtype, device=logits.device)
    _whole(out, logits.dtype, (T, E), "d_logits")
    queue = _queue(stream, logits, ids, weights, d_weights, out, status)
    p = _route_params(score, k, 1, 1, 1, renorm, scale)
    _check(lib().vp_route_grad(_ptr(logits), dt, T, E, ld, p, _ptr(ids), _ptr(weights), _ptr(d_weights),
                               _ptr(out), _ptr(status), queue), "vp_route_grad")
    return out


# --------------------------------------------------------------- experts

def expert_offsets(counts: torch.Tensor, self_rank: int, out: Optional[torch.Tensor] = None,
                   status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_expert_offsets: first row of each of rank self_rank's experts, int64 [E/N + 1], from counts [N, E]."""
    if counts.dim() != 2:
        raise ValueError("counts must be [N, E]")
    N, E = counts.shape
    _whole(counts, torch.int32, (N, E), "counts")
    n_local = E // max(N, 1)
    if out is None:
        out = _from(stream, torch.empty, n_local + 1, dtype=torch.int64, device=counts.device)
    _whole(out, torch.int64, (n_local + 1,), "offsets")
    queue = _queue(stream, counts, out, status)
    _check(lib().vp_expert_offsets(_ptr(counts), N, E, self_rank, _ptr(out), _ptr(status), queue),
           "vp_expert_offsets")
    return out


def _groups(offsets: torch.Tensor, n_local: int):
    _whole(offsets, torch.int64, (n_local + 1,), "offsets")


def _weights3(w: torch.Tensor, dtype, name: str = "w"):
    if w.dim() != 3:
        raise ValueError("%s must be [experts, rows, columns]" % name)
    _whole(w, dtype, w.shape, name)
    return w.shape


def expert_matmul(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, *, gated: bool = False,
                  out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                  status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_expert_matmul: y = x W_e^T for every expert's rows of x [R, K], w [L, N, K] bf16 or fp16; gated: y =
    silu(x G^T) * (x U^T) [R, N/2] with the halves G, U of W_e, which `pre` [R, N] takes before the gate."""
    dt = _float_dtype(x, "x", halves=True)
    L, N, K = _weights3(w, x.dtype)
    ldx = _matrix(x, "x", cols=K)
    R = x.shape[0]
    _groups(offsets, L)
    width = N // 2 if gated else N
    if out is None:
        out = _from(stream, torch.empty, (R, width), dtype=x.dtype, device=x.device)
    ldy = _matrix(out, "out", cols=width, dtype=x.dtype, rows=R)
    ldp = 0 if pre is None else _matrix(pre, "pre", cols=N, dtype=x.dtype, rows=R)
    queue = _queue(stream, x, w, offsets, out, pre, status)
    _check(lib().vp_expert_matmul(_ptr(x), 2 * ldx, dt, _ptr(w), _ptr(offsets), R, L, N, K, int(gated), _ptr(out),
                                  2 * ldy, _ptr(pre), 2 * ldp, _ptr(status), queue), "vp_expert_matmul")
    return out


def expert_matmul_grad_x(dy: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, *,
                         out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """vp_expert_matmul_grad_x: dx = dy W_e [R, K] for every expert's rows of dy [R, N]."""
    dt = _float_dtype(dy, "dy", halves=True)
    L, N, K = _weights3(w, dy.dtype)
    ldy = _matrix(dy, "dy", cols=N)
    R = dy.shape[0]
    _groups(offsets, L)
    if out is None:
        out = _from(stream, torch.empty, (R, K), dtype=dy.dtype, device=dy.device)
    ldx = _matrix(out, "out", cols=K, dtype=dy.dtype, rows=R)
    queue = _queue(stream, dy, w, offsets, out, status)
    _check(lib().vp_expert_matmul_grad_x(_ptr(dy), 2 * ldy, dt, _ptr(w), _ptr(offsets), R, L, N, K, _ptr(out),
                                         2 * ldx, _ptr(status), queue), "vp_expert_matmul_grad_x")
    return out


def expert_matmul_grad_w(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor, *,
                         out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """vp_expert_matmul_grad_w: dW_e = dy^T x over the expert's rows, fp32 [L, N, K]."""
    dt = _float_dtype(dy, "dy", halves=True)
    if dy.dim() != 2 or offsets.dim() != 1:
        raise ValueError("dy must be a matrix, offsets a vector")
    R, N = dy.shape
    ldy = _matrix(dy, "dy")
    ldx = _matrix(x, "x", dtype=dy.dtype, rows=R)
    K, L = x.shape[1], offsets.numel() - 1
    _groups(offsets, L)
    if out is None:
        out = _from(stream, torch.empty, (L, N, K), dtype=torch.float32, device=dy.device)
    _whole(out, torch.float32, (L, N, K), "out")
    queue = _queue(stream, dy, x, offsets, out, status)
    _check(lib().vp_expert_matmul_grad_w(_ptr(dy), 2 * ldy, _ptr(x), 2 * ldx, dt, _ptr(offsets), R, L, N, K,
                                         _ptr(out), _ptr(status), queue), "vp_expert_matmul_grad_w")
    return out


def expert_gate_grad(dh: torch.Tensor, pre: torch.Tensor, offsets: torch.Tensor, *,
                     out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """vp_expert_gate_grad: the gradient [R, 2 I] of silu(g) * u by pre = (g, u), from dh [R, I]."""
    dt = _float_dtype(dh, "dh", halves=True)
    ldh = _matrix(dh, "dh")
    R, half = dh.shape
    ldp = _matrix(pre, "pre", cols=2 * half, dtype=dh.dtype, rows=R)
    L = offsets.numel() - 1
    _groups(offsets, L)
    if out is None:
        out = _from(stream, torch.empty, (R, 2 * half), dtype=dh.dtype, device=dh.device)
    ldo = _matrix(out, "out", cols=2 * half, dtype=dh.dtype, rows=R)
    queue = _queue(stream, dh, pre, offsets, out, status)
    _check(lib().vp_expert_gate_grad(_ptr(dh), 2 * ldh, _ptr(pre), 2 * ldp, dt, _ptr(offsets), R, L, half, _ptr(out),
                                     2 * ldo, _ptr(status), queue), "vp_expert_gate_grad")
    return out


# ----------------------------------------------------------------- merge

def merge(rows: torch.Tensor, weights: torch.Tensor, *, residual: Optional[torch.Tensor] = None,
          out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_merge: out[t] = residual[t] + sum_j weights[t, j] rows[t k + j], rows [T k, H], weights fp32 [T, k]."""
    dt = _float_dtype(rows, "rows")
    if weights.dim() != 2:
        raise ValueError("weights must be [T, k]")
    T, k = weights.shape
    _whole(weights, torch.float32, (T, k), "weights")
    ldr = _matrix(rows, "rows", rows=T * k)
    H, size = rows.shape[1], rows.element_size()
    lds = 0 if residual is None else _matrix(residual, "residual", cols=H, dtype=rows.dtype, rows=T)
    if out is None:
        out = _from(stream, torch.empty, (T, H), dtype=rows.dtype, device=rows.device)
    ldo = _matrix(out, "out", cols=H, dtype=rows.dtype, rows=T)
    queue = _queue(stream, rows, weights, residual, out)
    _check(lib().vp_merge(_ptr(rows), dt, T, k, H, ldr * size, _ptr(weights), _ptr(residual), lds * size, _ptr(out),
                          ldo * size, queue), "vp_merge")
    return out


def merge_grad(d_out: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor, *,
               d_rows: Optional[torch.Tensor] = None, d_weights: Optional[torch.Tensor] = None, stream=None):
    """vp_merge_grad: (d_rows [T k, H], d_weights fp32 [T, k]); the residual's gradient is d_out itself."""
    dt = _float_dtype(rows, "rows")
    if weights.dim() != 2:
        raise ValueError("weights must be [T, k]")
    T, k = weights.shape
    _whole(weights, torch.float32, (T, k), "weights")
    ldr = _matrix(rows, "rows", rows=T * k)
    H, size = rows.shape[1], rows.element_size()
    ldd = _matrix(d_out, "d_out", cols=H, dtype=rows.dtype, rows=T)
    if d_rows is None:
        d_rows = _from(stream, torch.empty, (T * k, H), dtype=rows.dtype, device=rows.device)
    if d_weights is None:
        d_weights = _from(stream, torch.empty, (T, k), dtype=torch.float32, device=rows.device)
    ldo = _matrix(d_rows, "d_rows", cols=H, dtype=rows.dtype, rows=T * k)
    _whole(d_weights, torch.float32, (T, k), "d_weights")
    queue = _queue(stream, rows, d_out, weights, d_rows, d_weights)
    _check(lib().vp_merge_grad(_ptr(d_out), dt, T, k, H, ldd * size, _ptr(rows), ldr * size, _ptr(weights),
                               _ptr(d_rows), ldo * size, _ptr(d_weights), queue), "vp_merge_grad")
    return d_rows, d_weights


# --------------------------------------------------------- 4-bit blocks

def mx_row_bytes(K: int) -> int:
    """Bytes of a row of K values in 4-bit blocks (0 unless K is a positive multiple of 32)."""
    return int(lib().vp_mx_row_bytes(K))


def mx_quantize(x: torch.Tensor, *, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_mx_quantize: the last axis of x [..., K] in blocks of 32 values, uint8 [..., mx_row_bytes(K)].  A
    contiguous x may have any number of axes (an expert's weights [L, N, K]); a matrix may have strided rows."""
    dt = _float_dtype(x, "x")
    K = x.shape[-1] if x.dim() else 0
    if x.dim() != 2 and not x.is_contiguous():
        raise ValueError("x must be a matrix or contiguous")
    flat = x if x.dim() == 2 else x.reshape(-1, K)
    ldx = _matrix(flat, "x")
    rb = mx_row_bytes(K)
    if out is None:
        out = _from(stream, torch.empty, (*x.shape[:-1], rb), dtype=torch.uint8, device=x.device)
    if out.shape != (*x.shape[:-1], rb) or (out.dim() != 2 and not out.is_contiguous()):
        raise ValueError("out must be uint8 %s" % ((*x.shape[:-1], rb),))
    ldq = _matrix(out if out.dim() == 2 else out.view(-1, rb), "out", dtype=torch.uint8)
    queue = _queue(stream, x, out)
    _check(lib().vp_mx_quantize(_ptr(x), dt, flat.shape[0], K, ldx * x.element_size(), _ptr(out), ldq, queue),
           "vp_mx_quantize")
    return out


def mx_dequantize(q: torch.Tensor, K: int, *, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """vp_mx_dequantize: the values [R, K] that packed rows q [R, mx_row_bytes(K)] stand for."""
    ldq = _matrix(q, "q", cols=mx_row_bytes(K), dtype=torch.uint8)
    R = q.shape[0]
    if out is None:
        out = _from(stream, torch.empty, (R, K), dtype=dtype, device=q.device)
    dt = _float_dtype(out, "out")
    ldo = _matrix(out, "out", cols=K, rows=R)
    queue = _queue(stream, q, out)
    _check(lib().vp_mx_dequantize(_ptr(q), R, K, ldq, _ptr(out), dt, ldo * out.element_size(), queue),
           "vp_mx_dequantize")
    return out


def expert_matmul_mx(xq: torch.Tensor, wq: torch.Tensor, offsets: torch.Tensor, K: int, *, gated: bool = False,
                     dtype=torch.bfloat16, out: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vp_expert_matmul_mx: expert_matmul with rows xq [R, mx_row_bytes(K)] and weights wq [L, N, mx_row_bytes(K)]
    in 4-bit blocks; y is bf16 or fp16."""
    L, N, rb = _weights3(wq, torch.uint8, "wq")
    if rb != mx_row_bytes(K):
        raise ValueError("wq must hold rows of %d bytes" % mx_row_bytes(K))
    ldx = _matrix(xq, "xq", cols=rb, dtype=torch.uint8)
    R = xq.shape[0]
    _groups(offsets, L)
    width = N // 2 if gated else N
    if out is None:
        out = _from(stream, torch.empty, (R, width), dtype=dtype, device=xq.device)
    dt = _float_dtype(out, "out", halves=True)
    ldy = _matrix(out, "out", cols=width, rows=R)
    queue = _queue(stream, xq, wq, offsets, out, status)
    _check(lib().vp_expert_matmul_mx(_ptr(xq), ldx, _ptr(wq), _ptr(offsets), R, L, N, K, int(gated), _ptr(out), dt,
                                     2 * ldy, _ptr(status), queue), "vp_expert_matmul_mx")
    return out


# -------------------------------------------------------- kernels chosen

def expert_kernel(R: int, n_local: int, N: int, K: int, *, mode: str = "forward", gated: bool = False,
                  mx: bool = False) -> str:
    """vp_expert_kernel: "few_rows", "tiles_128" or "tiles_256", by which a product of these sizes is computed; mode
    "forward", "grad_x" or "grad_w"."""
    kind = lib().vp_expert_kernel(("forward", "grad_x", "grad_w").index(mode), int(mx), int(gated), R, n_local, N, K)
    if kind < 0:
        raise ValueError("no product has these sizes")
    return ("few_rows", "tiles_128", "tiles_256")[kind]


def route_lanes(T: int, E: int) -> int:
    """vp_route_lanes: how many lanes share a token of E experts' logits where T tokens are routed, 64 or 16."""
    lanes = int(lib().vp_route_lanes(T, E))
    if lanes < 0:
        raise ValueError("no routing has these sizes")
    return lanes
