"""Python binding of the student operators (``include/tabpack_ops.h``): gated
feed-forward block, RMS norm and layer norm, 8-bit product, distillation loss,
embedding lookup, dropout.

Argument checks and marshalling only.  Tensors are CUDA tensors, bf16 or
float32; rows may be spaced (any stride of the first dimension that is at
least the row's length), the last dimension is contiguous.  Work runs on
``stream`` (a torch stream; None: the current one), where outputs and
workspaces are also allocated, and is not waited for.  With ``stream`` the
inputs' memory is kept until that stream has read them, so that the caller may
let go of them at once; that they are written before it reads them, and
outputs before another stream does, is the caller's to order.

Nothing here takes part in autograd: outputs have no graph, whether or not an
input requires a gradient.  Gradients come from the ``_backward`` calls and from
``distill``, which returns its own; a caller that wants them in a graph wraps the
pairs in a ``torch.autograd.Function``.
"""
from __future__ import annotations

import ctypes
import functools
import threading

import torch

ACTIVATIONS = {"relu": 0, "silu": 1, "gelu": 2}
_PRECISION = {torch.bfloat16: 0, torch.float32: 1}
_empty = torch.empty

# A small call's time is the host's: entry points are looked up once, and a
# call takes no contexts, wrappers or imports on its way to the library.
_C = None


def _lib():
    """The library's entry points (loaded at the first call)."""
    global _C
    if _C is None:
        from . import load_library
        _C = load_library()
    return _C


def _fail(status):
    from . import _check
    _check(status)


def _precision(t, name):
    p = _PRECISION.get(t.dtype)
    if p is None:
        raise ValueError(f"{name}: expected bfloat16 or float32, got {t.dtype}")
    return p


_MAX_SIZE = (1 << 31) - 1   # of the library's 32-bit sizes, which ctypes would cut


def _too_wide(name, n):
    return ValueError(f"{name}: a width of {n} is not below 2^31")


def _elsewhere(t, name, device):
    """A call works on the device of its first tensor, which has to be the
    current one (_stream)."""
    return ValueError(f"{name}: expected a CUDA tensor on the call's device {device}, got device {t.get_device()}")


def _mat(t, name, device, dtype, rows=None, cols=None):
    """(pointer, row stride) of a matrix with contiguous rows."""
    if t.get_device() != device:
        raise _elsewhere(t, name, device)
    if t.dtype is not dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name}: shape {tuple(shape)}, expected ({'rows' if rows is None else rows}, "
                         f"{'columns' if cols is None else cols})")
    ld, one = t.stride()
    n = shape[1]
    if n > _MAX_SIZE:
        raise _too_wide(name, n)
    if one != 1 and n > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if ld < n or shape[0] <= 1:
        if shape[0] > 1:
            raise ValueError(f"{name}: rows overlap")
        ld = n
    return t.data_ptr(), ld


def _flat(t, name, device, dtype, *shape):
    """Pointer of a contiguous tensor of the given shape (None for None)."""
    if t is None:
        return None
    if t.get_device() != device:
        raise _elsewhere(t, name, device)
    if t.dtype is not dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(device):
    """The current stream's pointer; the call's device has to be the current one."""
    if device < 0 or device != _device():
        raise ValueError("expected CUDA tensors on the current device")
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(device)


def _on(stream, fn, tensors, *args):
    """fn(*tensors, *args) on another stream, which the allocator is told of."""
    with torch.cuda.stream(stream):
        out = fn(*tensors, *args)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return out


_local = threading.local()
_SMALL = 1 << 22


def _work(n, st, t):
    """(pointer, owner) of n bytes of workspace on t's device for a call on
    stream st.  Small ones of the default stream, which outlives every call and
    is never captured, are kept by the thread that uses them: an allocation is
    a tenth of a small call's time."""
    if st or n > _SMALL:
        w = _empty(n, dtype=torch.uint8, device=t.device)
        return w.data_ptr(), w
    space = _local.__dict__
    d = t.get_device()
    got = space.get(d)
    if got is None or got[0] < n:
        w = _empty(max(n, 1 << 16), dtype=torch.uint8, device=t.device)
        got = space[d] = (w.numel(), w.data_ptr(), w)
    return got[1], got[2]


@functools.lru_cache(maxsize=1024)
def _gated_bytes(rows, d, f, d_out, prec):
    v = [ctypes.c_int64() for _ in range(3)]
    status = _lib().pack_gated_bytes(rows, d, f, d_out, prec, *(ctypes.byref(x) for x in v))
    if status:
        _fail(status)
    return tuple(x.value for x in v)


def _gated_shapes(x, w_gate_up, w_down):
    prec, dtype, on = _precision(x, "x"), x.dtype, x.get_device()
    xp, ldx = _mat(x, "x", on, dtype)
    rows, d = x.shape
    gate, down = w_gate_up.shape, w_down.shape
    if len(gate) != 2 or gate[0] % 2 or len(down) != 2:
        raise ValueError("w_gate_up must be [2 f, d] and w_down [d_out, f]")
    f, d_out = gate[0] // 2, down[0]
    if f > _MAX_SIZE or d_out > _MAX_SIZE:
        raise _too_wide("w_gate_up or w_down", max(f, d_out))
    wp = _flat(w_gate_up, "w_gate_up", on, dtype, 2 * f, d)
    dp = _flat(w_down, "w_down", on, dtype, d_out, f)
    return prec, on, xp, ldx, rows, d, f, d_out, wp, dp


def gated_forward(x, w_gate_up, w_down, act="silu", save=False, stream=None):
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T with w_gate_up = [Wg; Wu] [2 f, d] and
    w_down [d_out, f].  save=True returns (y, saved) for gated_backward, the only
    way to its gradients (no autograd graph)."""
    if stream is not None:
        return _on(stream, gated_forward, (x, w_gate_up, w_down), act, save)
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    prec, on, xp, ldx, rows, d, f, d_out, wp, dp = _gated_shapes(x, w_gate_up, w_down)
    n_saved, n_work, _ = _gated_bytes(rows, d, f, d_out, prec)
    st, dev = _stream(on), x.device
    y = _empty((rows, d_out), dtype=x.dtype, device=dev)
    saved = _empty(n_saved, dtype=torch.uint8, device=dev) if save else None
    work, _keep = _work(n_work, st, x)
    status = _lib().pack_gated_forward(xp, ldx, wp, dp, rows, d, f, d_out, code, prec, y.data_ptr(),
                                       saved.data_ptr() if save else None, work, n_work, st)
    if status:
        _fail(status)
    return (y, saved) if save else y


def gated_backward(dy, x, w_gate_up, w_down, saved, stream=None):
    """(dx, dw_gate_up, dw_down) of the gated_forward call that saved."""
    if stream is not None:
        return _on(stream, gated_backward, (dy, x, w_gate_up, w_down, saved))
    prec, on, xp, ldx, rows, d, f, d_out, wp, dp = _gated_shapes(x, w_gate_up, w_down)
    gp, ldg = _mat(dy, "dy", on, x.dtype, rows, d_out)
    n_saved, _, n_work = _gated_bytes(rows, d, f, d_out, prec)
    sp = _flat(saved, "saved", on, torch.uint8, n_saved)
    st, dev = _stream(on), x.device
    dx = _empty((rows, d), dtype=x.dtype, device=dev)
    dw = _empty((2 * f, d), dtype=x.dtype, device=dev)
    dd = _empty((d_out, f), dtype=x.dtype, device=dev)
    work, _keep = _work(n_work, st, x)
    status = _lib().pack_gated_backward(gp, ldg, xp, ldx, wp, dp, sp, rows, d, f, d_out, prec, dx.data_ptr(),
                                        dw.data_ptr(), dd.data_ptr(), work, n_work, st)
    if status:
        _fail(status)
    return dx, dw, dd


def _norm(x, weight, residual, eps, q8):
    prec, dtype, on = _precision(x, "x"), x.dtype, x.get_device()
    xp, ldx = _mat(x, "x", on, dtype)
    rows, d = x.shape
    wp = _flat(weight, "weight", on, torch.float32, d)
    rp, ldr = (None, 0) if residual is None else _mat(residual, "residual", on, dtype, rows, d)
    st, dev = _stream(on), x.device
    if residual is None:
        total, tp = x, None
    else:
        total = _empty((rows, d), dtype=dtype, device=dev)
        tp = total.data_ptr()
    if q8:
        y = _empty((rows, d), dtype=torch.int8, device=dev)
        scale = _empty(rows, dtype=torch.float32, device=dev)
        status = _lib().pack_rms_norm(xp, ldx, rp, ldr, wp, rows, d, eps, prec, tp, None, y.data_ptr(), scale.data_ptr(),
                                      st)
        if status:
            _fail(status)
        return y, scale, total
    y = _empty((rows, d), dtype=dtype, device=dev)
    status = _lib().pack_rms_norm(xp, ldx, rp, ldr, wp, rows, d, eps, prec, tp, y.data_ptr(), None, None, st)
    if status:
        _fail(status)
    return y, total


def rms_norm(x, weight, residual=None, eps=1e-6, stream=None):
    """(y, s): the RMS norm y of s = x + residual (x itself without one) times
    weight [d] (float32), and s for the next residual and rms_norm_backward, the
    only way to its gradients (no autograd graph)."""
    if stream is not None:
        return _on(stream, rms_norm, (x, weight, residual), eps)
    return _norm(x, weight, residual, eps, False)


def rms_norm_q8(x, weight, residual=None, eps=1e-6, stream=None):
    """(q, scale, s): rms_norm with its output as int8 q [rows, d] and a scale
    per row, y = q * scale[:, None]."""
    if stream is not None:
        return _on(stream, rms_norm_q8, (x, weight, residual), eps)
    return _norm(x, weight, residual, eps, True)


@functools.lru_cache(maxsize=1024)
def _norm_bytes(rows, d):
    v = ctypes.c_int64()
    status = _lib().pack_rms_norm_bytes(rows, d, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def rms_norm_backward(dy, s, weight, dsum=None, eps=1e-6, stream=None):
    """(dx, dweight): gradients at s (= at x and at residual) and at weight;
    dsum: the gradient that reaches s from elsewhere, added to dx."""
    if stream is not None:
        return _on(stream, rms_norm_backward, (dy, s, weight, dsum), eps)
    prec, dtype, on = _precision(s, "s"), s.dtype, s.get_device()
    sp, lds = _mat(s, "s", on, dtype)
    rows, d = s.shape
    gp, ldg = _mat(dy, "dy", on, dtype, rows, d)
    wp = _flat(weight, "weight", on, torch.float32, d)
    ap, lda = _mat(dsum, "dsum", on, dtype, rows, d) if dsum is not None else (None, 0)
    n = _norm_bytes(rows, d)
    st, dev = _stream(on), s.device
    dx = _empty((rows, d), dtype=dtype, device=dev)
    dw = _empty(d, dtype=torch.float32, device=dev)
    work, _keep = _work(n, st, s)
    status = _lib().pack_rms_norm_backward(gp, ldg, sp, lds, wp, ap, lda, rows, d, eps, prec, dx.data_ptr(),
                                           dw.data_ptr(), work, n, st)
    if status:
        _fail(status)
    return dx, dw


@functools.lru_cache(maxsize=1024)
def _product_bytes(rows, k, n, prec):
    v = ctypes.c_int64()
    status = _lib().pack_product_q8_bytes(rows, k, n, prec, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def product_q8(q, scale, w, w_scale, bias=None, dtype=torch.bfloat16, stream=None):
    """y[r, c] = (sum_k q[r, k] w[c, k]) scale[r] w_scale[c] + bias[c]: q int8
    [rows, k], w int8 [n, k], scales and bias float32, y of type dtype."""
    if stream is not None:
        return _on(stream, product_q8, (q, scale, w, w_scale, bias), dtype)
    prec = _PRECISION.get(dtype)
    if prec is None:
        raise ValueError(f"dtype: expected bfloat16 or float32, got {dtype}")
    on = q.get_device()
    qp, ldq = _mat(q, "q", on, torch.int8)
    rows, k = q.shape
    if w.dim() != 2:
        raise ValueError("w must be [n, k]")
    n = w.shape[0]
    if n > _MAX_SIZE:
        raise _too_wide("w", n)
    wp = _flat(w, "w", on, torch.int8, n, k)
    sp = _flat(scale, "scale", on, torch.float32, rows)
    cp = _flat(w_scale, "w_scale", on, torch.float32, n)
    bp = _flat(bias, "bias", on, torch.float32, n)
    n_work = _product_bytes(rows, k, n, prec)
    st, dev = _stream(on), q.device
    y = _empty((rows, n), dtype=dtype, device=dev)
    work, _keep = _work(n_work, st, q) if n_work else (None, None)
    status = _lib().pack_product_q8(qp, ldq, sp, wp, cp, bp, rows, k, n, prec, y.data_ptr(),
                                    work, n_work, st)
    if status:
        _fail(status)
    return y


@functools.lru_cache(maxsize=1024)
def _distill_bytes(m, rows):
    v = ctypes.c_int64()
    status = _lib().pack_distill_bytes(m, rows, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def distill(z, ids, top, labels=None, tau=1.0, alpha=1.0, grad=True, stream=None):
    """(loss [m], dz or None): alpha times the tau^2-weighted divergence of each
    of m students from the teacher's top entries, plus 1 - alpha times the
    cross-entropy with labels, mean over the rows.  z [m, rows, n] (or
    [rows, n] for one student); ids int32 and top float32 [rows, k]: classes
    (-1: none) and logits of the teacher's entries; labels int32 [rows].  dz is the
    gradient of loss[i] at z[i] (no autograd graph)."""
    if stream is not None:
        return _on(stream, distill, (z, ids, top, labels), tau, alpha, grad)
    prec = _precision(z, "z")
    shape, on = z.shape, z.get_device()
    if len(shape) not in (2, 3) or not z.is_contiguous():
        raise ValueError("z must be a contiguous CUDA tensor [m, rows, n] or [rows, n]")
    m, rows, n = (1, *shape) if len(shape) == 2 else shape
    if ids.dim() != 2:
        raise ValueError("ids must be [rows, k]")
    k = ids.shape[1]
    if n > _MAX_SIZE or k > _MAX_SIZE:
        raise _too_wide("z or ids", max(n, k))
    ip = _flat(ids, "ids", on, torch.int32, rows, k)
    top_p = _flat(top, "top", on, torch.float32, rows, k)
    yp = _flat(labels, "labels", on, torch.int32, rows)
    n_work = _distill_bytes(m, rows)
    st, dev = _stream(on), z.device
    loss = _empty(m, dtype=torch.float32, device=dev)
    dz = torch.empty_like(z) if grad else None
    work, _keep = _work(n_work, st, z)
    status = _lib().pack_distill(z.data_ptr(), m, rows, n, ip, top_p, k, yp, tau, alpha, prec, loss.data_ptr(),
                                 dz.data_ptr() if grad else None, work, n_work, st)
    if status:
        _fail(status)
    return loss, dz


def _ids(ids, device):
    """(pointer, bytes an id, their number) of contiguous ids of any shape."""
    if ids.get_device() != device:
        raise _elsewhere(ids, "ids", device)
    size = _ID_BYTES.get(ids.dtype)
    if size is None:
        raise ValueError(f"ids: expected int32 or int64, got {ids.dtype}")
    if not ids.is_contiguous():
        raise ValueError("ids: expected a contiguous tensor")
    return ids.data_ptr(), size, ids.shape.numel()


_ID_BYTES = {torch.int32: 4, torch.int64: 8}


def _out_type(dtype, name="dtype"):
    p = _PRECISION.get(dtype)
    if p is None:
        raise ValueError(f"{name}: expected bfloat16 or float32, got {dtype}")
    return p


def embed(ids, table, scale=1.0, dtype=None, stream=None):
    """scale * table[ids], of shape [*ids.shape, d] and type dtype (None: the
    table's): ids int32 or int64, table [vocab, d].  An id outside 0..vocab-1
    (such as -1) gives zeros.  Gradients come from embed_backward (no autograd
    graph)."""
    if stream is not None:
        return _on(stream, embed, (ids, table), scale, dtype)
    prec, on = _precision(table, "table"), table.get_device()
    dtype = table.dtype if dtype is None else dtype
    out = _out_type(dtype)
    tp, ldt = _mat(table, "table", on, table.dtype)
    vocab, d = table.shape
    if vocab > _MAX_SIZE:
        raise _too_wide("table", vocab)
    ip, size, n = _ids(ids, on)
    st = _stream(on)
    y = _empty((*ids.shape, d), dtype=dtype, device=table.device)
    status = _lib().pack_embed(ip, size, n, tp, ldt, vocab, d, scale, prec, out, y.data_ptr(), st)
    if status:
        _fail(status)
    return y


@functools.lru_cache(maxsize=1024)
def _embed_bytes(n, vocab, d):
    v = ctypes.c_int64()
    status = _lib().pack_embed_bytes(n, vocab, d, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def embed_backward(dy, ids, vocab, scale=1.0, dtype=torch.float32, stream=None):
    """The gradient [vocab, d], of type dtype, at the table of embed(ids, table,
    scale): dy [*ids.shape, d], or [n, d] with spaced rows."""
    if stream is not None:
        return _on(stream, embed_backward, (dy, ids), vocab, scale, dtype)
    prec, on = _precision(dy, "dy"), dy.get_device()
    out = _out_type(dtype)
    ip, size, n = _ids(ids, on)
    if dy.dim() == 2 and dy.shape[0] == n:
        gp, ldg = _mat(dy, "dy", on, dy.dtype)
    elif dy.dim() and dy.shape[:-1] == ids.shape:
        gp, ldg = _flat(dy, "dy", on, dy.dtype, *dy.shape), dy.shape[-1]
    else:
        raise ValueError(f"dy: shape {tuple(dy.shape)}, expected (*ids.shape, d) of ids {tuple(ids.shape)}")
    d = dy.shape[-1]
    if max(vocab, d) > _MAX_SIZE:
        raise _too_wide("vocab or dy", max(vocab, d))
    n_work = _embed_bytes(n, vocab, d)
    st = _stream(on)
    dt = _empty((vocab, d), dtype=dtype, device=dy.device)
    work, _keep = _work(n_work, st, dy) if n_work else (None, None)
    status = _lib().pack_embed_backward(gp, ldg, ip, size, n, vocab, d, scale, prec, out, dt.data_ptr(), work, n_work, st)
    if status:
        _fail(status)
    return dt


def dropout(x, p, seed, step=0, site=0, residual=None, stream=None):
    """x [rows, d] with elements zeroed at rate p and the others over 1 - p, plus
    residual where one is given.  The mask is a function of (seed, step, site,
    row, column), as a pack's masks are: other steps and sites, other masks."""
    if stream is not None:
        return _on(stream, _dropout, (x, residual), p, seed, step, site)
    return _dropout(x, residual, p, seed, step, site)


def _dropout(x, residual, p, seed, step, site):
    prec, dtype, on = _precision(x, "x"), x.dtype, x.get_device()
    xp, ldx = _mat(x, "x", on, dtype)
    rows, d = x.shape
    rp, ldr = (None, 0) if residual is None else _mat(residual, "residual", on, dtype, rows, d)
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 32 and 0 <= site < 1 << 32):
        raise ValueError("seed must be of 64 bits, step and site of 32")
    st = _stream(on)
    y = _empty((rows, d), dtype=dtype, device=x.device)
    status = _lib().pack_dropout(xp, ldx, rp, ldr, rows, d, p, seed, step, site, prec, y.data_ptr(), st)
    if status:
        _fail(status)
    return y


def dropout_backward(dy, p, seed, step=0, site=0, stream=None):
    """The gradient at x of dropout(x, p, seed, step, site): the same elements of
    dy over 1 - p.  (The gradient at residual is dy.)"""
    return dropout(dy, p, seed, step, site, None, stream)


def layer_norm(x, weight, bias=None, residual=None, eps=1e-5, save=False, stream=None):
    """(y, s): the layer norm y of s = x + residual (rounded to their type; x
    itself without one) times weight [d], plus bias [d] (float32), and s for the
    next residual.  save=True returns (y, s, stats) with what
    layer_norm_backward needs, the only way to its gradients (no autograd
    graph)."""
    if stream is not None:
        return _on(stream, layer_norm, (x, weight, bias, residual), eps, save)
    prec, dtype, on = _precision(x, "x"), x.dtype, x.get_device()
    xp, ldx = _mat(x, "x", on, dtype)
    rows, d = x.shape
    wp = _flat(weight, "weight", on, torch.float32, d)
    bp = _flat(bias, "bias", on, torch.float32, d)
    rp, ldr = (None, 0) if residual is None else _mat(residual, "residual", on, dtype, rows, d)
    st, dev = _stream(on), x.device
    if residual is None:
        total, tp = x, None
    else:
        total = _empty((rows, d), dtype=dtype, device=dev)
        tp = total.data_ptr()
    y = _empty((rows, d), dtype=dtype, device=dev)
    stats = _empty((rows, 2), dtype=torch.float32, device=dev) if save else None
    status = _lib().pack_layer_norm(xp, ldx, rp, ldr, wp, bp, rows, d, eps, prec, tp, y.data_ptr(),
                                    stats.data_ptr() if save else None, st)
    if status:
        _fail(status)
    return (y, total, stats) if save else (y, total)


@functools.lru_cache(maxsize=1024)
def _layer_norm_bytes(rows, d):
    v = ctypes.c_int64()
    status = _lib().pack_layer_norm_bytes(rows, d, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def layer_norm_backward(dy, s, weight, stats, dsum=None, stream=None):
    """(dx, dweight, dbias) of the layer_norm call that returned s and stats: dx
    is the gradient at s (= at x and at residual); dsum: the gradient that
    reaches s from elsewhere, added to dx."""
    if stream is not None:
        return _on(stream, layer_norm_backward, (dy, s, weight, stats, dsum))
    prec, dtype, on = _precision(s, "s"), s.dtype, s.get_device()
    sp, lds = _mat(s, "s", on, dtype)
    rows, d = s.shape
    gp, ldg = _mat(dy, "dy", on, dtype, rows, d)
    wp = _flat(weight, "weight", on, torch.float32, d)
    mp = _flat(stats, "stats", on, torch.float32, rows, 2)
    ap, lda = _mat(dsum, "dsum", on, dtype, rows, d) if dsum is not None else (None, 0)
    n = _layer_norm_bytes(rows, d)
    st, dev = _stream(on), s.device
    dx = _empty((rows, d), dtype=dtype, device=dev)
    dw = _empty(d, dtype=torch.float32, device=dev)
    db = _empty(d, dtype=torch.float32, device=dev)
    work, _keep = _work(n, st, s)
    status = _lib().pack_layer_norm_backward(gp, ldg, sp, lds, wp, mp, ap, lda, rows, d, prec, dx.data_ptr(), dw.data_ptr(),
                                             db.data_ptr(), work, n, st)
    if status:
        _fail(status)
    return dx, dw, db


def quantise_f8(x, block_rows=1, stream=None):
    """(q, scale): x [rows, k] as float8_e4m3fn with a float32 scale [ceil(rows /
    block_rows), ceil(k / 128)] for every 128 columns of a row (block_rows=1:
    activations) or of 128 rows (block_rows=128: weights).  q's rows are padded to
    multiples of 16 bytes, as product_f8 takes them best."""
    if stream is not None:
        return _on(stream, quantise_f8, (x,), block_rows)
    prec, on = _precision(x, "x"), x.get_device()
    xp, ldx = _mat(x, "x", on, x.dtype)
    if block_rows not in (1, 128):
        raise ValueError(f"block_rows must be 1 or 128, not {block_rows}")
    rows, k = x.shape
    st, dev = _stream(on), x.device
    ldq = (k + 15) // 16 * 16
    q = _empty((rows, ldq), dtype=torch.float8_e4m3fn, device=dev)
    scale = _empty(((rows + block_rows - 1) // block_rows, (k + 127) // 128), dtype=torch.float32, device=dev)
    status = _lib().pack_quantise_f8(xp, ldx, rows, k, block_rows, prec, q.data_ptr(), ldq, scale.data_ptr(), st)
    if status:
        _fail(status)
    return q if ldq == k else q.as_strided((rows, k), (ldq, 1)), scale


@functools.lru_cache(maxsize=1024)
def _f8_bytes(rows, k, n, aligned):
    v = ctypes.c_int64()
    status = _lib().pack_product_f8_bytes(rows, k, n, aligned, ctypes.byref(v))
    if status:
        _fail(status)
    return v.value


def product_f8(q, scale, w, w_scale, bias=None, dtype=torch.bfloat16, stream=None):
    """y[r, c] = sum_b scale[r, b] w_scale[c // 128, b] sum_{k in block b} q[r, k]
    w[c, k] + bias[c], of type dtype: q [rows, k] and scale of quantise_f8, w
    [n, k] and w_scale of quantise_f8(weights, 128), bias float32 [n].  Operands
    whose rows do not start at multiples of 16 bytes are copied first."""
    if stream is not None:
        return _on(stream, product_f8, (q, scale, w, w_scale, bias), dtype)
    prec = _out_type(dtype)
    on = q.get_device()
    qp, ldq = _mat(q, "q", on, torch.float8_e4m3fn)
    rows, k = q.shape
    if w.dim() != 2:
        raise ValueError("w must be [n, k]")
    n = w.shape[0]
    if n > _MAX_SIZE:
        raise _too_wide("w", n)
    wp, ldw = _mat(w, "w", on, torch.float8_e4m3fn, n, k)
    blocks = (k + 127) // 128
    sp = _flat(scale, "scale", on, torch.float32, rows, blocks)
    cp = _flat(w_scale, "w_scale", on, torch.float32, (n + 127) // 128, blocks)
    bp = _flat(bias, "bias", on, torch.float32, n)
    odd = qp | wp | (ldq if rows > 1 else 0) | (ldw if n > 1 else 0)   # (one row has no distance to the next)
    n_work = _f8_bytes(rows, k, n, odd & 15 == 0)
    st, dev = _stream(on), q.device
    y = _empty((rows, n), dtype=dtype, device=dev)
    work, _keep = _work(n_work, st, q) if n_work else (None, None)
    status = _lib().pack_product_f8(qp, ldq, sp, wp, ldw, cp, bp, rows, k, n, prec, y.data_ptr(), work, n_work, st)
    if status:
        _fail(status)
    return y


def ops_check(stream=None):
    """Waits for the stream; raises if a bounded wait of a product has given up on
    this device since the calling thread's last check of this stream."""
    status = _lib().pack_ops_check((stream or torch.cuda.current_stream()).cuda_stream)
    if status:
        _fail(status)
