"""Thin ctypes binding of libdeamoe.so: argument marshalling only.

Every step of the layer runs in the library's CUDA kernels.  torch is used here for device
memory (tensors handed in by the caller) and for the current stream, nothing else.  If the
library has not been built the import of `lib()` raises -- there is no fallback.
"""
import ctypes as C
import os

import torch


_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdeamoe.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALLOC, ERR_CUDA, ERR_BATCH, ERR_TIMEOUT, ERR_INTERNAL = range(8)
DENSE_MIN_BATCH = 32   # calls of this many tokens and more take the dense schedule under SCHED_AUTO (csrc/dense.cuh) ...
DENSE_SMALL_ROUTER = 64  # ... twice as many on layers of fewer experts than this

F32, BF16 = 0, 1
SIGMA_NONE, SIGMA_SILU, SIGMA_GELU, SIGMA_RMSNORM = 0, 1, 2, 3
SCHED_AUTO, SCHED_PLAIN, SCHED_STAGED, SCHED_FUSED, SCHED_DENSE = 0, 1, 2, 3, 4


def dense_min_batch(shape):
    """Smallest call that SCHED_AUTO runs in the dense schedule on a layer of this shape (if it supports it)."""
    n = shape.n_dept * shape.experts_per_dept
    return DENSE_MIN_BATCH if n >= DENSE_SMALL_ROUTER else 2 * DENSE_MIN_BATCH


# every symbol include/deamoe.h declares
SYMBOLS = ("deamoe_layer_create", "deamoe_vanilla_create", "deamoe_layer_destroy", "deamoe_route",
           "deamoe_forward", "deamoe_vanilla_forward", "deamoe_forward_host", "deamoe_forward_partial",
           "deamoe_finish_partial", "deamoe_get_routing",
           "deamoe_get_stats", "deamoe_profile_enable", "deamoe_profile_last_ms", "deamoe_route_static", "deamoe_failure_test", "deamoe_probe_read",
           "deamoe_last_launches", "deamoe_device_bytes", "deamoe_status_string",
           "deamoe_sort_workspace", "deamoe_sort_pairs", "deamoe_dispatch", "deamoe_dispatch_backward", "deamoe_combine",
           "deamoe_combine_backward", "deamoe_norm_workspace", "deamoe_norm", "deamoe_norm_backward",
           "deamoe_norm_residual", "deamoe_norm_residual_backward", "deamoe_quant_workspace", "deamoe_quant_product")

GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = 0, 1, 2, 3


class Config(C.Structure):
    _fields_ = [(k, C.c_int32) for k in (
        "hidden", "n_dept", "experts_per_dept", "ffn", "priv", "top_k", "k_dept", "n_shared",
        "shared_ffn", "sigma", "norm_topk", "weight_dtype", "act_dtype", "residual", "max_batch",
        "schedule")] + [("route_scale", C.c_float), ("strict_dept", C.c_int32), ("dept_begin", C.c_int32),
                        ("dept_end", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in (
        "router", "dept_gate", "dept_up", "dept_down", "priv_gate", "priv_up", "priv_down",
        "shared_gate", "shared_up", "shared_down")]


class DeaMoEError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib():
    """Load libdeamoe.so (built in-tree by build.py); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2608_14385_b200.build` "
                              "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        for name in SYMBOLS:
            getattr(L, name)
        L.deamoe_status_string.restype = C.c_char_p
        L.deamoe_status_string.argtypes = [C.c_int]
        L.deamoe_last_launches.restype = C.c_int32
        L.deamoe_last_launches.argtypes = [C.c_void_p]
        L.deamoe_device_bytes.restype = C.c_uint64
        L.deamoe_device_bytes.argtypes = [C.c_void_p]
        for name in ("deamoe_layer_create", "deamoe_vanilla_create"):
            getattr(L, name).argtypes = [C.POINTER(Config), C.POINTER(Weights), C.c_void_p,
                                         C.POINTER(C.c_void_p)]
        L.deamoe_layer_destroy.argtypes = [C.c_void_p]
        L.deamoe_route.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        for name in ("deamoe_forward", "deamoe_vanilla_forward", "deamoe_forward_host"):
            getattr(L, name).argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.deamoe_forward_partial.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.deamoe_finish_partial.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.deamoe_get_routing.argtypes = [C.c_void_p] * 9
        L.deamoe_get_stats.argtypes = [C.c_void_p] * 7
        L.deamoe_route_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                          C.c_int32, C.c_int32, C.c_float, C.c_int32, C.c_void_p, C.c_void_p]
        L.deamoe_failure_test.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        L.deamoe_probe_read.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
        L.deamoe_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        L.deamoe_profile_last_ms.argtypes = [C.c_void_p, C.POINTER(C.c_float)]
        i, l, u, f, p = C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_void_p
        for name, res, args in (
                ("deamoe_sort_workspace", u, (i, i, i)),
                ("deamoe_sort_pairs", i, (p, p, i, i, i, p, p, p, p, u)),
                ("deamoe_dispatch", i, (p, i, p, l, p, i, i, i, p, l, l)),
                ("deamoe_dispatch_backward", i, (p, i, p, l, l, p, i, i, i, p, l)),
                ("deamoe_combine", i, (p, i, p, l, l, p, p, i, i, i, p, l)),
                ("deamoe_combine_backward", i, (p, i, p, l, p, l, l, p, p, i, i, i, p, l, p)),
                ("deamoe_norm_workspace", u, (i, i)),
                ("deamoe_norm", i, (p, i, p, l, i, i, i, p, f, p, l)),
                ("deamoe_norm_backward", i, (p, i, p, l, i, i, i, p, f, p, l, p, l, p, l, p, p, u)),
                ("deamoe_norm_residual", i, (p, i, p, l, p, l, i, i, i, i, p, f, i, p, l, f, f, p, l, p, f, p, l)),
                ("deamoe_norm_residual_backward", i, (p, i, p, l, p, l, i, i, i, i, p, f, i, p, l, f, f, p, l, p, f, p, l,
                                                      p, l, p, l, p, l, p, p, p, u)),
                ("deamoe_quant_workspace", u, (i, i, i)),
                ("deamoe_quant_product", i, (p, i, p, i, p, p, i, i, i, i, p, l, i, p, p, i, i, i, p, l, p, u))):
            getattr(L, name).restype = res
            getattr(L, name).argtypes = args
        _lib = L
    return _lib


def status_string(status):
    return lib().deamoe_status_string(int(status)).decode()


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def make_config(shape, max_batch, schedule=SCHED_AUTO, dept_range=None):
    d = shape.asdict() if hasattr(shape, "asdict") else dict(shape)
    lo, hi = dept_range if dept_range is not None else (0, 0)
    return Config(d["hidden"], d["n_dept"], d["experts_per_dept"], d["ffn"], d["priv"], d["top_k"],
                  d.get("k_dept", 0), d.get("n_shared", 0), d.get("shared_ffn", 0), d.get("sigma", 1),
                  d.get("norm_topk", 1), d.get("weight_dtype", 1), d.get("act_dtype", 1),
                  d.get("residual", 0), int(max_batch), int(schedule), float(d.get("route_scale", 1.0)),
                  int(d.get("strict_dept", 0)), int(lo), int(hi))


STATIC_ROUTE_SCRATCH_BYTES = 4 << 20
PROBE_BLOCKS = 2368


def probe_read(buf, sink):
    """Enqueue one plain read of the CUDA tensor `buf` (deamoe_probe_read); sink: int32 CUDA tensor of
    at least PROBE_BLOCKS elements.  The caller times it with events."""
    assert buf.is_cuda and buf.is_contiguous() and sink.is_cuda and sink.numel() >= PROBE_BLOCKS
    st = lib().deamoe_probe_read(_stream(), _dptr(buf), buf.numel() * buf.element_size(), _dptr(sink))
    if st != OK:
        raise DeaMoEError(st, "deamoe_probe_read")



def route_static(router, tokens, n_dept, experts_per_dept, top_k, norm_topk=1, route_scale=1.0, idx=None, w=None):
    """Allocation-free routing (deamoe_route_static): for hosts that cannot create a layer object
    because they may not allocate device memory (graph capture, latency-critical loops, plug-ins
    working inside someone else's memory pool).  router [n, h] and tokens [B, h] are fp32 CUDA
    tensors; idx [B, k] int32 and w [B, k] fp32 are caller-provided outputs (made here only when
    omitted, for convenience in tests).  All calls share one fixed scratch array inside the library:
    do not overlap two calls on the GPU."""
    assert router.is_cuda and tokens.is_cuda and router.dtype == torch.float32 and tokens.dtype == torch.float32
    B, h = tokens.shape
    if idx is None:
        idx = torch.empty((B, top_k), dtype=torch.int32, device=tokens.device)
    if w is None:
        w = torch.empty((B, top_k), dtype=torch.float32, device=tokens.device)
    st = lib().deamoe_route_static(_stream(), _dptr(router), _dptr(tokens), n_dept, experts_per_dept, h, top_k,
                                   norm_topk, float(route_scale), B, _dptr(idx), _dptr(w))
    if st != OK:
        raise DeaMoEError(st, "deamoe_route_static")
    return idx, w


# ---------------------------------------------------------------- operators around a layer
# Thin wrappers like the rest of this file: they check what the C call cannot see (types, shapes, the device a tensor
# lives on), make outputs and workspaces that were not handed in, and call.  Matrices may have any row stride.

_TYPES = {torch.float32: F32, torch.bfloat16: BF16}
_INT_MAX = 2 ** 31 - 1  # sizes beyond it would reach the library without their upper bits


def _refuse(where, why):
    e = DeaMoEError(ERR_INVALID_ARG, where)
    e.args = (f"{e.args[0]}: {why}",)
    raise e


_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _raw_stream(device):
    """The current stream's handle (a decode step's calls are short: torch.cuda.current_stream builds an object first)."""
    return torch.cuda.current_stream(device).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    _raw_stream = torch._C._cuda_getCurrentRawStream


def _mat(t, where, name, dtype, rows, cols, dev):
    """Address and row stride of a [rows, cols] matrix of device `dev`, the current one."""
    if t.dtype is not dtype or t.shape != (rows, cols):
        _refuse(where, f"{name} must be {dtype} [{rows}, {cols}], got {t.dtype} {list(t.shape)}")
    if t.get_device() != dev:
        _refuse(where, f"{name} is not on the current CUDA device")
    if rows > _INT_MAX or cols > _INT_MAX:
        _refuse(where, f"{name} [{rows}, {cols}] has a side of 2^31 or more")
    stride, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(where, f"{name} must have consecutive values in a row")
    return t.data_ptr(), stride if rows > 1 else cols


def _vec(t, where, name, dtype, shape, dev):
    """Address of a contiguous array of device `dev`, the current one."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(where, f"{name} must be contiguous {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
    if t.get_device() != dev:
        _refuse(where, f"{name} is not on the current CUDA device")
    return t.data_ptr()


def _type(t, where, name):
    code = _TYPES.get(t.dtype)
    if code is None or t.dim() != 2:
        _refuse(where, f"{name} must be a float32 or bfloat16 matrix, got {t.dtype} {list(t.shape)}")
    return code


def _pairs(pair_row, where):
    if pair_row.dim() != 2:
        _refuse(where, f"pair_row must be [T, k], got {list(pair_row.shape)}")
    if pair_row.shape[1] > _INT_MAX:
        _refuse(where, "top_k of 2^31 or more")
    return pair_row.shape


def _workspace(nbytes, like):
    """Scratch of one call: from torch's allocator on the current stream (a captured graph's own pool while capturing),
    so no two calls share it unless the stream orders them."""
    return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _done(status, where):
    if status != OK:
        raise DeaMoEError(status, where)


def sort_pairs(topk_idx, n_expert):
    """(token, slot) pairs in expert order (deamoe_sort_pairs).  topk_idx: int32 [T, k], as Layer.route gives it; entries
    outside [0, n_expert) drop their pair.  Returns expert_off [n_expert + 1], pair_row [T, k] (-1 = dropped) and
    row_pair [T * k] (-1 behind the last row), all int32."""
    where, dev = "deamoe_sort_pairs", _device()
    if topk_idx.dim() != 2:
        _refuse(where, "topk_idx must be [T, k]")
    T, k = topk_idx.shape
    src = _vec(topk_idx, where, "topk_idx", torch.int32, (T, k), dev)
    n = int(n_expert)
    if not 0 < n <= _INT_MAX or T > _INT_MAX or k > _INT_MAX:
        _refuse(where, f"{T} tokens, top_k {k}, {n} experts")
    off = topk_idx.new_empty(n + 1)
    pair_row = topk_idx.new_empty((T, k))
    row_pair = topk_idx.new_empty(T * k)
    L = lib()
    need = L.deamoe_sort_workspace(T, k, n)
    ws = _workspace(need, topk_idx)
    _done(L.deamoe_sort_pairs(_raw_stream(dev), src, T, k, n, off.data_ptr(), pair_row.data_ptr(), row_pair.data_ptr(),
                              _ptr(ws), need), where)
    return off, pair_row, row_pair


def dispatch(x, pair_row, rows=None):
    """rows[pair_row[t, q]] = x[t] (deamoe_dispatch).  rows: [n_rows, h] to fill; made with T * k rows if omitted (rows
    that no pair points to are then uninitialised)."""
    where, dev = "deamoe_dispatch", _device()
    dt = _type(x, where, "x")
    T, h = x.shape
    k = _pairs(pair_row, where)[1]
    if rows is None:
        rows = x.new_empty((T * k, h))
    n = rows.shape[0]
    px, sx = _mat(x, where, "x", x.dtype, T, h, dev)
    pr, sr = _mat(rows, where, "rows", x.dtype, n, h, dev)
    _done(lib().deamoe_dispatch(_raw_stream(dev), dt, px, sx, _vec(pair_row, where, "pair_row", torch.int32, (T, k), dev), T, k, h, pr, sr,
                                n), where)
    return rows


def dispatch_backward(drows, pair_row, dx=None):
    """dx[t] = sum_q drows[pair_row[t, q]] (deamoe_dispatch_backward)."""
    where, dev = "deamoe_dispatch_backward", _device()
    dt = _type(drows, where, "drows")
    n, h = drows.shape
    T, k = _pairs(pair_row, where)
    if dx is None:
        dx = drows.new_empty((T, h))
    pd, sd = _mat(drows, where, "drows", drows.dtype, n, h, dev)
    px, sx = _mat(dx, where, "dx", drows.dtype, T, h, dev)
    _done(lib().deamoe_dispatch_backward(_raw_stream(dev), dt, pd, sd, n, _vec(pair_row, where, "pair_row", torch.int32, (T, k), dev), T, k,
                                         h, px, sx), where)
    return dx


def combine(rows, pair_row, topk_w, out=None):
    """out[t] = sum_q topk_w[t, q] rows[pair_row[t, q]] (deamoe_combine)."""
    where, dev = "deamoe_combine", _device()
    dt = _type(rows, where, "rows")
    n, h = rows.shape
    T, k = _pairs(pair_row, where)
    if out is None:
        out = rows.new_empty((T, h))
    pr, sr = _mat(rows, where, "rows", rows.dtype, n, h, dev)
    po, so = _mat(out, where, "out", rows.dtype, T, h, dev)
    _done(lib().deamoe_combine(_raw_stream(dev), dt, pr, sr, n, _vec(pair_row, where, "pair_row", torch.int32, (T, k), dev),
                               _vec(topk_w, where, "topk_w", torch.float32, (T, k), dev), T, k, h, po, so), where)
    return out


def combine_backward(dout, rows, pair_row, topk_w, drows=None, dw=None):
    """drows[pair_row[t, q]] = topk_w[t, q] dout[t] and dw[t, q] = <dout[t], rows[pair_row[t, q]]>
    (deamoe_combine_backward).  Returns (drows, dw); rows of drows that no pair points to are left as they were
    (uninitialised if drows was made here)."""
    where, dev = "deamoe_combine_backward", _device()
    dt = _type(dout, where, "dout")
    T, h = dout.shape
    k = _pairs(pair_row, where)[1]
    if rows.dim() != 2:
        _refuse(where, f"rows must be a matrix, got {list(rows.shape)}")
    n = rows.shape[0]
    if drows is None:
        drows = dout.new_empty((n, h))
    if dw is None:
        dw = dout.new_empty((T, k), dtype=torch.float32)
    pd, sd = _mat(dout, where, "dout", dout.dtype, T, h, dev)
    pr, sr = _mat(rows, where, "rows", dout.dtype, n, h, dev)
    pg, sg = _mat(drows, where, "drows", dout.dtype, n, h, dev)
    _done(lib().deamoe_combine_backward(_raw_stream(dev), dt, pd, sd, pr, sr, n, _vec(pair_row, where, "pair_row", torch.int32, (T, k), dev),
                                        _vec(topk_w, where, "topk_w", torch.float32, (T, k), dev), T, k, h, pg, sg,
                                        _vec(dw, where, "dw", torch.float32, (T, k), dev)), where)
    return drows, dw


def _gain(w, where, name, h, dev, other=None):
    """Address and type code of a gain (None = ones).  Two gains of one call have one type."""
    if w is None:
        return None, (F32 if other is None else _TYPES.get(other.dtype, -1))
    code = _TYPES.get(w.dtype)
    if code is None or (other is not None and other.dtype != w.dtype):
        _refuse(where, f"{name} must be float32 or bfloat16, and of one type with the call's other gain")
    return _vec(w, where, name, w.dtype, (h,), dev), code


def norm(x, weight, eps, out=None):
    """out = x / sqrt(mean(x^2) + eps) * weight, row by row (deamoe_norm).  weight [h] (float32 or bfloat16) or None; out may
    be x."""
    where, dev = "deamoe_norm", _device()
    dt = _type(x, where, "x")
    T, h = x.shape
    if out is None:
        out = torch.empty_like(x)
    px, sx = _mat(x, where, "x", x.dtype, T, h, dev)
    po, so = _mat(out, where, "out", x.dtype, T, h, dev)
    pw, wdt = _gain(weight, where, "weight", h, dev)
    _done(lib().deamoe_norm(_raw_stream(dev), dt, px, sx, T, h, wdt, pw, eps, po, so), where)
    return out


def norm_backward(x, weight, eps, du, dadd=None, dx=None):
    """Gradients of `norm`: dx (plus dadd, the gradient that reaches x past the norm; dx may be dadd) and dweight
    (float32 [h]) (deamoe_norm_backward)."""
    where, dev = "deamoe_norm_backward", _device()
    dt = _type(x, where, "x")
    T, h = x.shape
    if dx is None:
        dx = torch.empty_like(x)
    dw = x.new_empty(h, dtype=torch.float32)
    px, sx = _mat(x, where, "x", x.dtype, T, h, dev)
    pu, su = _mat(du, where, "du", x.dtype, T, h, dev)
    pa, sa = _mat(dadd, where, "dadd", x.dtype, T, h, dev) if dadd is not None else (None, 0)
    pd, sd = _mat(dx, where, "dx", x.dtype, T, h, dev)
    pw, wdt = _gain(weight, where, "weight", h, dev)
    L = lib()
    need = L.deamoe_norm_workspace(T, h)
    ws = _workspace(need, x)
    _done(L.deamoe_norm_backward(_raw_stream(dev), dt, px, sx, T, h, wdt, pw, eps, pu, su, pa, sa, pd, sd, dw.data_ptr(), _ptr(ws),
                                 need), where)
    return dx, dw


def _gate(gate, where, dtype, T, h, kind, dev):
    """Kind, address and row stride of a gate.  [h] is one per channel, [T, 1] or [T] one per token, [T, h] full; a gate of
    one dimension with T == h needs `gate_kind` (and [T, 1] with h == 1 is full without it)."""
    if gate is None:
        return GATE_NONE, None, 0
    shape = tuple(gate.shape)
    if kind is None:
        if len(shape) == 1 and T == h and shape == (h,):
            _refuse(where, "gate [h] with as many tokens as channels: say gate_kind")
        kind = {(h,): GATE_CHANNEL, (T,): GATE_TOKEN, (T, 1): GATE_TOKEN, (T, h): GATE_FULL}.get(shape)
    if kind == GATE_FULL:
        return (kind,) + _mat(gate, where, "gate", dtype, T, h, dev)
    if kind not in (GATE_CHANNEL, GATE_TOKEN):
        _refuse(where, f"gate must be [{h}] (channels), [{T}] or [{T}, 1] (tokens) or [{T}, {h}], got {list(shape)}")
    want = (h,) if kind == GATE_CHANNEL else shape if shape == (T, 1) else (T,)
    return kind, _vec(gate, where, "gate", dtype, want, dev), 0


def norm_residual(x, y, weight, eps, gate=None, residual_scale=1.0, branch_scale=1.0, normalise=True, next_norm=True,
                  next_weight=None, next_eps=None, gate_kind=None, out=None, next_out=None):
    """s = residual_scale x + branch_scale gate (y / rms(y) weight); returns s and s / rms(s) next_weight (None with
    next_norm=False) in one pass (deamoe_norm_residual).  gate: None, [h], [T], [T, 1] or [T, h]; normalise=False takes y as it
    is.  out may be x."""
    where, dev = "deamoe_norm_residual", _device()
    dt = _type(x, where, "x")
    T, h = x.shape
    if out is None:
        out = torch.empty_like(x)
    if next_out is None and next_norm:
        next_out = torch.empty_like(x)
    px, sx = _mat(x, where, "x", x.dtype, T, h, dev)
    py, sy = _mat(y, where, "y", x.dtype, T, h, dev)
    po, so = _mat(out, where, "out", x.dtype, T, h, dev)
    pn, sn = _mat(next_out, where, "next_out", x.dtype, T, h, dev) if next_norm else (None, 0)
    pw, wdt = _gain(weight, where, "weight", h, dev, next_weight)
    pm, _ = _gain(next_weight, where, "next_weight", h, dev, weight)
    kind, pg, sg = _gate(gate, where, x.dtype, T, h, gate_kind, dev)
    _done(lib().deamoe_norm_residual(_raw_stream(dev), dt, px, sx, py, sy, T, h, 1 if normalise else 0, wdt, pw, eps, kind, pg, sg,
                                     residual_scale, branch_scale, po, so, pm, eps if next_eps is None else next_eps,
                                     pn, sn), where)
    return out, next_out if next_norm else None


def norm_residual_backward(x, y, weight, eps, dout, gate=None, residual_scale=1.0, branch_scale=1.0, normalise=True,
                           next_weight=None, next_eps=None, du=None, gate_kind=None, dx=None, dy=None):
    """Gradients of `norm_residual` from those of its outputs (dout, and du of the next norm or None): dx, dy, dgate,
    dweight, dnext_weight; the last three are None where the call has no such input.  dweight, dnext_weight and the
    gradient of a per-channel or per-token gate are float32, that of a full gate has the gate's type; dgate has the gate's
    shape (deamoe_norm_residual_backward)."""
    where, dev = "deamoe_norm_residual_backward", _device()
    dt = _type(x, where, "x")
    T, h = x.shape
    if dx is None:
        dx = torch.empty_like(x)
    if dy is None:
        dy = torch.empty_like(x)
    px, sx = _mat(x, where, "x", x.dtype, T, h, dev)
    py, sy = _mat(y, where, "y", x.dtype, T, h, dev)
    po, so = _mat(dout, where, "dout", x.dtype, T, h, dev)
    pu, su = _mat(du, where, "du", x.dtype, T, h, dev) if du is not None else (None, 0)
    pdx, sdx = _mat(dx, where, "dx", x.dtype, T, h, dev)
    pdy, sdy = _mat(dy, where, "dy", x.dtype, T, h, dev)
    pw, wdt = _gain(weight, where, "weight", h, dev, next_weight)
    pm, _ = _gain(next_weight, where, "next_weight", h, dev, weight)
    kind, pg, sg = _gate(gate, where, x.dtype, T, h, gate_kind, dev)
    dgate, sdg = None, 0
    channel = kind == GATE_CHANNEL
    n = (weight is not None) + (next_weight is not None) + channel
    sums = list(x.new_empty((n, h), dtype=torch.float32).unbind(0)) if n else []
    dw = sums.pop() if weight is not None else None
    dn = sums.pop() if next_weight is not None else None
    if channel:
        dgate = sums.pop()
    elif kind == GATE_TOKEN:
        dgate = x.new_empty(gate.shape, dtype=torch.float32)
    elif kind == GATE_FULL:
        dgate, sdg = x.new_empty((T, h)), h
    L = lib()
    need = L.deamoe_norm_workspace(T, h)
    ws = _workspace(need, x)
    _done(L.deamoe_norm_residual_backward(_raw_stream(dev), dt, px, sx, py, sy, T, h, 1 if normalise else 0, wdt, pw, eps, kind, pg,
                                          sg, residual_scale, branch_scale, po, so, pm,
                                          eps if next_eps is None else next_eps, pu, su, pdx, sdx, pdy, sdy, _ptr(dgate),
                                          sdg, _ptr(dw), _ptr(dn), _ptr(ws), need), where)
    return dx, dy, dgate, dw, dn


def quant_product(codes, scales, x, group, zeros=None, expert_off=None, row_pair=None, pairs_per_token=1, swiglu=False,
                  out=None):
    """Products with 4-bit matrices (deamoe_quant_product): codes uint8 [E, n_out, n_in / 2] (low four bits first),
    scales (float32 or bfloat16) and zeros (uint8, None = 8) [E, n_out, ceil(n_in / group)], x [T, n_in].
    expert_off / row_pair: as sort_pairs gives them; row r is a product with x[row_pair[r] // pairs_per_token].  Without
    row_pair, row r takes x[r].  Rows behind the last expert's are left as they were (uninitialised if out was made here)."""
    where, dev = "deamoe_quant_product", _device()
    dt = _type(x, where, "x")
    T, n_in = x.shape
    if codes.dim() != 3 or n_in != 2 * codes.shape[2]:
        _refuse(where, f"codes must be [E, n_out, {n_in} / 2], got {list(codes.shape)}")
    E, n_out, _ = codes.shape
    if group not in (32, 64, 128) or not 0 < pairs_per_token <= _INT_MAX or E > _INT_MAX or n_out > _INT_MAX:
        _refuse(where, f"group {group} (32, 64 or 128), pairs_per_token {pairs_per_token}, {E} matrices of {n_out} rows")
    groups = -(-n_in // group)
    R = T if row_pair is None else row_pair.shape[0]
    width = n_out // 2 if swiglu else n_out
    if out is None:
        out = x.new_empty((R, width))
    sdt = _TYPES.get(scales.dtype)
    if sdt is None:
        _refuse(where, "scales must be float32 or bfloat16")
    px, sx = _mat(x, where, "x", x.dtype, T, n_in, dev)
    po, so = _mat(out, where, "out", x.dtype, R, width, dev)
    pz = _vec(zeros, where, "zeros", torch.uint8, (E, n_out, groups), dev) if zeros is not None else None
    pe = _vec(expert_off, where, "expert_off", torch.int32, (E + 1,), dev) if expert_off is not None else None
    pp = _vec(row_pair, where, "row_pair", torch.int32, (R,), dev) if row_pair is not None else None
    L = lib()
    need = L.deamoe_quant_workspace(dt, R, n_in)
    ws = _workspace(need, x)
    _done(L.deamoe_quant_product(_raw_stream(dev), dt, _vec(codes, where, "codes", torch.uint8, (E, n_out, n_in // 2), dev), sdt,
                                 _vec(scales, where, "scales", scales.dtype, (E, n_out, groups), dev), pz, E, n_out, n_in, group, px,
                                 sx, T, pe, pp, pairs_per_token, R, 1 if swiglu else 0, po, so, _ptr(ws), need), where)
    return out


class Layer:
    """One DeaMoE (or vanilla MoE) layer living on the current CUDA device."""

    def __init__(self, shape, weights, max_batch, schedule=SCHED_AUTO, vanilla=False, dept_range=None):
        """weights: dict of CUDA tensors in the canonical layouts of include/deamoe.h.
        dept_range = (begin, end): this object is the slice of the layer holding those departments
        (the dept_* / priv_* tensors then hold only them); use forward_partial / finish_partial."""
        self.shape = shape
        self.vanilla = vanilla
        self.cfg = make_config(shape, max_batch, schedule, dept_range)
        if vanilla:
            self.cfg.priv = 0
        w = Weights()
        for name, _ in Weights._fields_:
            t = weights.get(name)
            if vanilla and name.startswith("priv_"):
                t = None
            if t is not None:
                assert t.is_cuda and t.is_contiguous(), name
            setattr(w, name, t.data_ptr() if t is not None else None)
        self._h = C.c_void_p()
        fn = lib().deamoe_vanilla_create if vanilla else lib().deamoe_layer_create
        st = fn(C.byref(self.cfg), C.byref(w), _stream(), C.byref(self._h))
        if st != OK:
            self._h = C.c_void_p()
            raise DeaMoEError(st, "deamoe_vanilla_create" if vanilla else "deamoe_layer_create")
        self.act = torch.float32 if self.cfg.act_dtype == F32 else torch.bfloat16

    def close(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.deamoe_layer_destroy(h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check_tokens(self, tokens):
        assert tokens.is_cuda and tokens.is_contiguous() and tokens.dtype == self.act
        assert tokens.dim() == 2 and tokens.shape[1] == self.cfg.hidden
        return tokens.shape[0]

    def route(self, tokens, want_outputs=True):
        B = self._check_tokens(tokens)
        k = self.cfg.top_k
        idx = torch.empty((B, k), dtype=torch.int32, device=tokens.device) if want_outputs else None
        w = torch.empty((B, k), dtype=torch.float32, device=tokens.device) if want_outputs else None
        st = lib().deamoe_route(self._h, _stream(), _dptr(tokens), B, _dptr(idx), _dptr(w))
        if st != OK:
            raise DeaMoEError(st, "deamoe_route")
        return idx, w

    def forward(self, tokens, out=None):
        B = self._check_tokens(tokens)
        if out is None:
            out = torch.empty_like(tokens)
        fn = lib().deamoe_vanilla_forward if self.vanilla else lib().deamoe_forward
        st = fn(self._h, _stream(), _dptr(tokens), B, _dptr(out))
        if st != OK:
            raise DeaMoEError(st, "deamoe_forward")
        return out

    def forward_partial(self, tokens, partial=None):
        """fp32 partial sum of this layer object (a department slice, or a whole layer): [B, h]."""
        B = self._check_tokens(tokens)
        if partial is None:
            partial = torch.empty(tokens.shape, dtype=torch.float32, device=tokens.device)
        assert partial.is_cuda and partial.is_contiguous() and partial.dtype == torch.float32
        st = lib().deamoe_forward_partial(self._h, _stream(), _dptr(tokens), B, _dptr(partial))
        if st != OK:
            raise DeaMoEError(st, "deamoe_forward_partial")
        return partial

    def finish_partial(self, total, tokens, out=None):
        """out = total (+ tokens if residual) in the activation dtype; total: the slices' partial sums added."""
        B = self._check_tokens(tokens)
        if out is None:
            out = torch.empty_like(tokens)
        assert total.is_cuda and total.is_contiguous() and total.dtype == torch.float32
        st = lib().deamoe_finish_partial(self._h, _stream(), _dptr(total), _dptr(tokens), B, _dptr(out))
        if st != OK:
            raise DeaMoEError(st, "deamoe_finish_partial")
        return out

    def forward_host(self, tokens, out):
        """tokens/out: CPU tensors (pinned for speed) [B, h] in the activation dtype."""
        assert not tokens.is_cuda and not out.is_cuda and tokens.is_contiguous() and out.is_contiguous()
        st = lib().deamoe_forward_host(self._h, _stream(), C.c_void_p(tokens.data_ptr()), tokens.shape[0],
                                       C.c_void_p(out.data_ptr()))
        if st != OK:
            raise DeaMoEError(st, "deamoe_forward_host")
        return out

    def routing(self, B):
        """Host copy of the last call's routing state as numpy arrays."""
        import numpy as np
        m, n, k = self.cfg.n_dept, self.cfg.n_dept * self.cfg.experts_per_dept, self.cfg.top_k
        idx = np.zeros((B, k), np.int32)
        w = np.zeros((B, k), np.float32)
        mask = np.zeros(((m + 63) // 64,), np.uint64)
        doff = np.zeros((m + 1,), np.int32)
        dtok = np.full((max(1, B * min(k, m)),), -1, np.int32)
        eoff = np.zeros((n + 1,), np.int32)
        etok = np.full((max(1, B * k),), -1, np.int32)
        st = lib().deamoe_get_routing(self._h, _stream(), *(C.c_void_p(a.ctypes.data)
                                                           for a in (idx, w, mask, doff, dtok, eoff, etok)))
        if st != OK:
            raise DeaMoEError(st, "deamoe_get_routing")
        return {"idx": idx, "w": w, "dept_mask": mask, "dept_off": doff, "dept_tok": dtok[:doff[m]],
                "expert_off": eoff, "expert_tok": etok[:eoff[n]]}

    def stats(self):
        nd, ne, ntd, st_ = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
        ub = C.c_uint64()
        st = lib().deamoe_get_stats(self._h, _stream(), C.byref(nd), C.byref(ne), C.byref(ntd), C.byref(ub),
                                    C.byref(st_))
        if st != OK:
            raise DeaMoEError(st, "deamoe_get_stats")
        return {"active_dept": nd.value, "active_expert": ne.value, "token_dept_pairs": ntd.value,
                "unique_weight_bytes": ub.value, "device_status": st_.value}

    def failure_test(self, wait_limit=0, withhold=0):
        """Test aid (deamoe_failure_test): lower the poll limit of the bounded device-side waits
        and / or withhold a hand-over so that a wait expires; (0, 0) restores normal operation."""
        st = lib().deamoe_failure_test(self._h, int(wait_limit), int(withhold))
        if st != OK:
            raise DeaMoEError(st, "deamoe_failure_test")

    def profile(self, enable=True):
        """Record CUDA events around the weight-streaming launches of later forward calls."""
        st = lib().deamoe_profile_enable(self._h, 1 if enable else 0)
        if st != OK:
            raise DeaMoEError(st, "deamoe_profile_enable")

    def last_stream_ms(self):
        """Milliseconds between those events for the last forward (synchronises on it)."""
        ms = C.c_float()
        st = lib().deamoe_profile_last_ms(self._h, C.byref(ms))
        if st != OK:
            raise DeaMoEError(st, "deamoe_profile_last_ms")
        return ms.value

    @property
    def last_launches(self):
        return lib().deamoe_last_launches(self._h)

    @property
    def device_bytes(self):
        return lib().deamoe_device_bytes(self._h)
