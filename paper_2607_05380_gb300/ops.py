"""Python binding of the student operators (``include/tabpack_ops.h``): gated
feed-forward block, RMS norm, 8-bit product, distillation loss.

Argument checks and marshalling only.  Tensors are CUDA tensors, bf16 or
float32; rows may be spaced (any stride of the first dimension that is at
least the row's length), the last dimension is contiguous.  Work runs on
``stream`` (a torch stream; None: the current one), where outputs and
workspaces are also allocated, and is not waited for.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

import torch

ACTIVATIONS = {"relu": 0, "silu": 1, "gelu": 2}
_PRECISION = {torch.bfloat16: 0, torch.float32: 1}


def _lib():
    from . import load_library
    return load_library()


def _ok(status):
    from . import _check
    _check(status)


def _precision(t, name):
    p = _PRECISION.get(t.dtype)
    if p is None:
        raise ValueError(f"{name}: expected bfloat16 or float32, got {t.dtype}")
    return p


def _mat(t, name, dtype, rows=None, cols=None, dims=2):
    """(pointer, row stride) of a matrix with contiguous rows."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.dim() != dims or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[-1] != cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({'rows' if rows is None else rows}, "
                         f"{'columns' if cols is None else cols})")
    n = t.shape[1]
    if n > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    ld = t.stride(0) if t.shape[0] > 1 else n
    if ld < n:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _flat(t, name, dtype, shape):
    """Pointer of a contiguous tensor of the given shape (None for None)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


def _on(stream, t):
    """(context for allocations, stream pointer) of a call on t's device."""
    if t.device.index != torch.cuda.current_device():
        raise ValueError("the tensors are not on the current device")
    if stream is None:
        return contextlib.nullcontext(), torch.cuda.current_stream().cuda_stream
    return torch.cuda.stream(stream), stream.cuda_stream


def _space(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _ptr(t):
    return None if t is None else t.data_ptr()


@functools.lru_cache(maxsize=1024)
def _gated_bytes(rows, d, f, d_out, prec):
    v = [ctypes.c_int64() for _ in range(3)]
    _ok(_lib().pack_gated_bytes(rows, d, f, d_out, prec, *(ctypes.byref(x) for x in v)))
    return tuple(x.value for x in v)


def _gated_shapes(x, w_gate_up, w_down):
    prec = _precision(x, "x")
    xp, ldx = _mat(x, "x", x.dtype)
    rows, d = x.shape
    if w_gate_up.dim() != 2 or w_gate_up.shape[0] % 2 or w_down.dim() != 2:
        raise ValueError("w_gate_up must be [2 f, d] and w_down [d_out, f]")
    f, d_out = w_gate_up.shape[0] // 2, w_down.shape[0]
    wp = _flat(w_gate_up, "w_gate_up", x.dtype, (2 * f, d))
    dp = _flat(w_down, "w_down", x.dtype, (d_out, f))
    return prec, xp, ldx, rows, d, f, d_out, wp, dp


def gated_forward(x, w_gate_up, w_down, act="silu", save=False, stream=None):
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T with w_gate_up = [Wg; Wu] [2 f, d] and
    w_down [d_out, f].  save=True returns (y, saved) for gated_backward."""
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    prec, xp, ldx, rows, d, f, d_out, wp, dp = _gated_shapes(x, w_gate_up, w_down)
    n_saved, n_work, _ = _gated_bytes(rows, d, f, d_out, prec)
    ctx, st = _on(stream, x)
    with ctx:
        y = torch.empty((rows, d_out), dtype=x.dtype, device=x.device)
        saved = torch.empty(n_saved, dtype=torch.uint8, device=x.device) if save else None
        work = _space(n_work, x.device)
    _ok(_lib().pack_gated_forward(xp, ldx, wp, dp, rows, d, f, d_out, ACTIVATIONS[act], prec, y.data_ptr(),
                                  _ptr(saved) if rows else None, _ptr(work), n_work, st))
    return (y, saved) if save else y


def gated_backward(dy, x, w_gate_up, w_down, saved, stream=None):
    """(dx, dw_gate_up, dw_down) of the gated_forward call that saved."""
    prec, xp, ldx, rows, d, f, d_out, wp, dp = _gated_shapes(x, w_gate_up, w_down)
    gp, ldg = _mat(dy, "dy", x.dtype, rows, d_out)
    n_saved, _, n_work = _gated_bytes(rows, d, f, d_out, prec)
    _flat(saved, "saved", torch.uint8, (n_saved,))
    ctx, st = _on(stream, x)
    with ctx:
        dx = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        dw = torch.empty_like(w_gate_up)
        dd = torch.empty_like(w_down)
        work = _space(n_work, x.device)
    _ok(_lib().pack_gated_backward(gp, ldg, xp, ldx, wp, dp, saved.data_ptr() if rows else None, rows, d, f, d_out, prec,
                                   dx.data_ptr(), dw.data_ptr(), dd.data_ptr(), _ptr(work), n_work, st))
    return dx, dw, dd


def _norm(x, weight, residual, eps, q8, stream):
    prec = _precision(x, "x")
    xp, ldx = _mat(x, "x", x.dtype)
    rows, d = x.shape
    wp = _flat(weight, "weight", torch.float32, (d,))
    rp, ldr = _mat(residual, "residual", x.dtype, rows, d) if residual is not None else (None, 0)
    ctx, st = _on(stream, x)
    with ctx:
        total = torch.empty((rows, d), dtype=x.dtype, device=x.device) if residual is not None else None
        if q8:
            y = torch.empty((rows, d), dtype=torch.int8, device=x.device)
            scale = torch.empty(rows, dtype=torch.float32, device=x.device)
        else:
            y, scale = torch.empty((rows, d), dtype=x.dtype, device=x.device), None
    yp = y.data_ptr()
    _ok(_lib().pack_rms_norm(xp, ldx, rp, ldr, wp, rows, d, eps, prec, _ptr(total), None if q8 else yp,
                             yp if q8 else None, _ptr(scale), st))
    return y, scale, x if residual is None else total


def rms_norm(x, weight, residual=None, eps=1e-6, stream=None):
    """(y, s): the RMS norm y of s = x + residual (x itself without one) times
    weight [d] (float32), and s for the next residual and rms_norm_backward."""
    y, _, s = _norm(x, weight, residual, eps, False, stream)
    return y, s


def rms_norm_q8(x, weight, residual=None, eps=1e-6, stream=None):
    """(q, scale, s): rms_norm with its output as int8 q [rows, d] and a scale
    per row, y = q * scale[:, None]."""
    return _norm(x, weight, residual, eps, True, stream)


@functools.lru_cache(maxsize=1024)
def _norm_bytes(rows, d):
    v = ctypes.c_int64()
    _ok(_lib().pack_rms_norm_bytes(rows, d, ctypes.byref(v)))
    return v.value


def rms_norm_backward(dy, s, weight, dsum=None, eps=1e-6, stream=None):
    """(dx, dweight): gradients at s (= at x and at residual) and at weight;
    dsum: the gradient that reaches s from elsewhere, added to dx."""
    prec = _precision(s, "s")
    sp, lds = _mat(s, "s", s.dtype)
    rows, d = s.shape
    gp, ldg = _mat(dy, "dy", s.dtype, rows, d)
    wp = _flat(weight, "weight", torch.float32, (d,))
    ap, lda = _mat(dsum, "dsum", s.dtype, rows, d) if dsum is not None else (None, 0)
    n = _norm_bytes(rows, d)
    ctx, st = _on(stream, s)
    with ctx:
        dx = torch.empty((rows, d), dtype=s.dtype, device=s.device)
        dw = torch.empty(d, dtype=torch.float32, device=s.device)
        work = _space(n, s.device)
    _ok(_lib().pack_rms_norm_backward(gp, ldg, sp, lds, wp, ap, lda, rows, d, eps, prec, dx.data_ptr(), dw.data_ptr(),
                                      _ptr(work), n, st))
    return dx, dw


@functools.lru_cache(maxsize=1024)
def _product_bytes(rows, k, n, prec):
    v = ctypes.c_int64()
    _ok(_lib().pack_product_q8_bytes(rows, k, n, prec, ctypes.byref(v)))
    return v.value


def product_q8(q, scale, w, w_scale, bias=None, dtype=torch.bfloat16, stream=None):
    """y[r, c] = (sum_k q[r, k] w[c, k]) scale[r] w_scale[c] + bias[c]: q int8
    [rows, k], w int8 [n, k], scales and bias float32, y of type dtype."""
    if dtype not in _PRECISION:
        raise ValueError(f"dtype: expected bfloat16 or float32, got {dtype}")
    prec = _PRECISION[dtype]
    qp, ldq = _mat(q, "q", torch.int8)
    rows, k = q.shape
    if w.dim() != 2:
        raise ValueError("w must be [n, k]")
    n = w.shape[0]
    wp = _flat(w, "w", torch.int8, (n, k))
    sp = _flat(scale, "scale", torch.float32, (rows,))
    cp = _flat(w_scale, "w_scale", torch.float32, (n,))
    bp = _flat(bias, "bias", torch.float32, (n,))
    n_work = _product_bytes(rows, k, n, prec)
    ctx, st = _on(stream, q)
    with ctx:
        y = torch.empty((rows, n), dtype=dtype, device=q.device)
        work = _space(n_work, q.device)
    _ok(_lib().pack_product_q8(qp, ldq, sp, wp, cp, bp, rows, k, n, prec, y.data_ptr(), _ptr(work), n_work, st))
    return y


@functools.lru_cache(maxsize=1024)
def _distill_bytes(m, rows):
    v = ctypes.c_int64()
    _ok(_lib().pack_distill_bytes(m, rows, ctypes.byref(v)))
    return v.value


def distill(z, ids, top, labels=None, tau=1.0, alpha=1.0, grad=True, stream=None):
    """(loss [m], dz or None): alpha times the tau^2-weighted divergence of each
    of m students from the teacher's top entries, plus 1 - alpha times the
    cross-entropy with labels, mean over the rows.  z [m, rows, n] (or
    [rows, n] for one student); ids int32 and top float32 [rows, k]: classes
    (-1: none) and logits of the teacher's entries; labels int32 [rows]."""
    prec = _precision(z, "z")
    if z.dim() not in (2, 3) or not z.is_cuda or not z.is_contiguous():
        raise ValueError("z must be a contiguous CUDA tensor [m, rows, n] or [rows, n]")
    m, rows, n = (1, *z.shape) if z.dim() == 2 else z.shape
    if ids.dim() != 2:
        raise ValueError("ids must be [rows, k]")
    k = ids.shape[1]
    ip = _flat(ids, "ids", torch.int32, (rows, k))
    tp_ = _flat(top, "top", torch.float32, (rows, k))
    yp = _flat(labels, "labels", torch.int32, (rows,))
    n_work = _distill_bytes(m, rows)
    ctx, st = _on(stream, z)
    with ctx:
        loss = torch.empty(m, dtype=torch.float32, device=z.device)
        dz = torch.empty_like(z) if grad else None
        work = _space(n_work, z.device)
    _ok(_lib().pack_distill(z.data_ptr(), m, rows, n, ip, tp_, k, yp, tau, alpha, prec, loss.data_ptr(), _ptr(dz),
                            _ptr(work), n_work, st))
    return loss, dz


def ops_check(stream=None):
    """Waits for the stream; raises if a bounded wait of a product gave up."""
    _ok(_lib().pack_ops_check((stream or torch.cuda.current_stream()).cuda_stream))
