"""Binding of include/ffn.h: the gated feed-forward block, the norms around it
with gate and residual scale, and counter-based dropout.

As in the package itself: the functions carry the C names and take device
pointers and a HIP stream; ``FfnPlan``, ``NormPlan`` and ``dropout`` take and
return CUDA (HIP) torch tensors.  Outputs and workspaces that the caller does
not give are allocated here, for the stream that uses them.
"""
from __future__ import annotations

import ctypes
import operator

FFN_FP32, FFN_BF16, FFN_FP16 = 0, 2, 3
FFN_SILU, FFN_GELU, FFN_RELU = 0, 1, 2
FFN_MAX_WIDTH, FFN_MAX_ROWS = 1 << 20, 1 << 30
__all__ = ["FFN_FP32", "FFN_BF16", "FFN_FP16", "FFN_SILU", "FFN_GELU", "FFN_RELU", "FFN_MAX_WIDTH", "FFN_MAX_ROWS",
           "ffn_norm", "ffn_plan", "ffn_destroy", "ffn_workspace_bytes", "ffn_backward_workspace_bytes", "ffn_forward",
           "ffn_backward", "ffn_norm_forward", "ffn_norm_backward", "ffn_norm_workspace_bytes", "ffn_residual_forward",
           "ffn_residual_backward", "ffn_dropout", "FfnPlan", "NormPlan", "dropout"]
_DTYPES = {"fp32": FFN_FP32, "bf16": FFN_BF16, "fp16": FFN_FP16}
_ACTIVATIONS = {"silu": FFN_SILU, "gelu": FFN_GELU, "relu": FFN_RELU}


class ffn_norm(ctypes.Structure):
    _fields_ = [("width", ctypes.c_int64), ("rows_per_gate", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("eps", ctypes.c_float), ("dropout", ctypes.c_double), ("seed", ctypes.c_uint64),
                ("offset", ctypes.c_uint64)]


_i32, _i64, _u64, _vp, _int = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int
_np = ctypes.POINTER(ffn_norm)
SIGNATURES = {
    "ffn_plan": (_int, [_i64, _i64, _i64, _i32, _i32, ctypes.POINTER(_vp)]),
    "ffn_destroy": (_int, [_vp]),
    "ffn_workspace_bytes": (_i64, [_vp, _i64]),
    "ffn_backward_workspace_bytes": (_i64, [_vp, _i64]),
    "ffn_forward": (_int, [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "ffn_backward": (_int, [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "ffn_norm_forward": (_int, [_np, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp]),
    "ffn_norm_backward": (_int, [_np, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp]),
    "ffn_residual_forward": (_int, [_np] + [_vp] * 9 + [_i64, _vp]),
    "ffn_residual_backward": (_int, [_np] + [_vp] * 15 + [_i64, _vp, _i64, _vp]),
    "ffn_norm_workspace_bytes": (_i64, [_np, _i64, _i32]),
    "ffn_dropout": (_int, [_vp, _i64, _vp, _i64, _i64, _i64, _i32, ctypes.c_double, _u64, _u64, _vp]),
}


_fn = {}   # entry points by name, once the library is loaded


def _entry(name):
    f = _fn.get(name)
    if f is None:
        from . import _load
        f = _fn[name] = getattr(_load(), name)
    return f


def _call(name, *args):
    rc = _entry(name)(*args)
    if rc:
        from . import _check
        _check(rc, name)


def _code(table, value, what):
    if value in table:
        return table[value]
    if isinstance(value, int):
        return value
    raise ValueError("%s must be one of %s" % (what, ", ".join(table)))


# ---------------------------------------------------------------- C names

def ffn_plan(d_in: int, d_ff: int, d_out: int, activation="silu", dtype="fp32") -> ctypes.c_void_p:
    h = ctypes.c_void_p()
    _call("ffn_plan", int(d_in), int(d_ff), int(d_out), _code(_ACTIVATIONS, activation, "activation"),
          _code(_DTYPES, dtype, "dtype"), ctypes.byref(h))
    return h


def ffn_destroy(plan) -> None:
    _call("ffn_destroy", plan)


def ffn_workspace_bytes(plan, N: int) -> int:
    return _entry("ffn_workspace_bytes")(plan, N)


def ffn_backward_workspace_bytes(plan, N: int) -> int:
    return _entry("ffn_backward_workspace_bytes")(plan, N)


def ffn_forward(plan, x_ptr, ldx, w_in_ptr, w_out_ptr, y_ptr, saved_ptr, N, ws_ptr, ws_bytes, stream_ptr=None) -> None:
    _call("ffn_forward", plan, x_ptr, ldx, w_in_ptr, w_out_ptr, y_ptr, saved_ptr, N, ws_ptr, ws_bytes, stream_ptr)


def ffn_backward(plan, x_ptr, ldx, w_in_ptr, w_out_ptr, saved_ptr, g_ptr, ldg, gx_ptr, gw_in_ptr, gw_out_ptr, N,
                 ws_ptr, ws_bytes, stream_ptr=None) -> None:
    _call("ffn_backward", plan, x_ptr, ldx, w_in_ptr, w_out_ptr, saved_ptr, g_ptr, ldg, gx_ptr, gw_in_ptr, gw_out_ptr,
          N, ws_ptr, ws_bytes, stream_ptr)


def ffn_norm_forward(norm, x_ptr, ldx, w_ptr, u_ptr, ldu, rstd_ptr, N, stream_ptr=None) -> None:
    _call("ffn_norm_forward", norm, x_ptr, ldx, w_ptr, u_ptr, ldu, rstd_ptr, N, stream_ptr)


def ffn_norm_backward(norm, x_ptr, ldx, w_ptr, rstd_ptr, gu_ptr, ldg, gx_ptr, gw_ptr, N, ws_ptr, ws_bytes,
                      stream_ptr=None) -> None:
    _call("ffn_norm_backward", norm, x_ptr, ldx, w_ptr, rstd_ptr, gu_ptr, ldg, gx_ptr, gw_ptr, N, ws_ptr, ws_bytes,
          stream_ptr)


def ffn_norm_workspace_bytes(norm, N: int, residual: int) -> int:
    return _entry("ffn_norm_workspace_bytes")(norm, N, residual)


def ffn_residual_forward(norm, x_ptr, h_ptr, w_ptr, gate_ptr, scale_ptr, w_next_ptr, y_ptr, u_ptr, stats_ptr, N,
                         stream_ptr=None) -> None:
    _call("ffn_residual_forward", norm, x_ptr, h_ptr, w_ptr, gate_ptr, scale_ptr, w_next_ptr, y_ptr, u_ptr, stats_ptr,
          N, stream_ptr)


def ffn_residual_backward(norm, h_ptr, y_ptr, w_ptr, gate_ptr, scale_ptr, w_next_ptr, stats_ptr, gy_ptr, gu_ptr,
                          gx_ptr, gh_ptr, gw_ptr, ggate_ptr, gscale_ptr, gw_next_ptr, N, ws_ptr, ws_bytes,
                          stream_ptr=None) -> None:
    _call("ffn_residual_backward", norm, h_ptr, y_ptr, w_ptr, gate_ptr, scale_ptr, w_next_ptr, stats_ptr, gy_ptr,
          gu_ptr, gx_ptr, gh_ptr, gw_ptr, ggate_ptr, gscale_ptr, gw_next_ptr, N, ws_ptr, ws_bytes, stream_ptr)


def ffn_dropout(x_ptr, ldx, y_ptr, ldy, N, width, dtype, p, seed, offset, stream_ptr=None) -> None:
    _call("ffn_dropout", x_ptr, ldx, y_ptr, ldy, N, width, _code(_DTYPES, dtype, "dtype"), p, seed, offset, stream_ptr)


# ---------------------------------------------------------------- convenience

def _word(n):
    """A whole number of any kind (those of numpy among them) modulo 2^64."""
    return operator.index(n) & 0xFFFFFFFFFFFFFFFF


class _Torch:
    """What the calls below need of torch, imported with the first of them."""

    def __getattr__(self, name):
        import torch
        self.empty_like, self.float32, self.uint8 = torch.empty_like, torch.float32, torch.uint8
        self.raw_stream, self.on_stream = torch._C._cuda_getCurrentRawStream, torch.cuda.stream
        self.current_device = torch._C._cuda_getDevice
        self.dtypes = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
        self.codes = {t: _DTYPES[name] for name, t in self.dtypes.items()}
        return self.__dict__[name]


_t = _Torch()


def _rows(t, tdt, rows, width, what, dev=None):
    """Row stride of t, which must be a [rows, width] tensor on GPU `dev` whose rows do not overlap (None: any)."""
    if not t.is_cuda or t.dtype != tdt or t.dim() != 2 or t.shape[1] != width or (rows is not None and t.shape[0] != rows):
        raise ValueError("%s must be a %s CUDA tensor [%s, %d]" % (what, tdt, "N" if rows is None else rows, width))
    if dev is not None and t.get_device() != dev:
        raise ValueError("all tensors must be on GPU %d: %s is not" % (dev, what))
    ld, one = t.stride()
    if t.shape[0] <= 1:   # (a stride that is never taken)
        ld = width
    if (width > 1 and one != 1) or ld < width:
        raise ValueError("%s must have adjacent values in each row and rows that do not overlap" % what)
    return ld


def _whole(t, tdt, shape, what, dev):
    """Pointer of t, a contiguous tensor of this shape on GPU `dev` (None where t is None)."""
    if t is None:
        return None
    if t.dtype != tdt or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor %s on GPU %d" % (what, tdt, list(shape), dev))
    return t.data_ptr()


def _stream(stream, dev):
    """The HIP stream's handle, and the torch stream where it is not the current one.  Kernels start on the current
    device, which must be the tensors'."""
    if _t.current_device() != dev:
        raise ValueError("the tensors are on GPU %d, which is not the current device" % dev)
    if stream is None:
        return _t.raw_stream(dev), None
    if stream.device_index != dev:
        raise ValueError("the stream is not one of GPU %d" % dev)
    return stream.cuda_stream, stream


def _new(t, shape, other):
    """A new tensor of t's type and device, of the stream `other` (None: the current one), so that its memory is reused
    in that stream's order."""
    if other is None:
        return t.new_empty(shape)
    with _t.on_stream(other):
        return t.new_empty(shape)


def _new32(t, shape, other):
    """The same, of 32-bit floats."""
    if t.dtype == _t.float32:
        return _new(t, shape, other)
    if other is None:
        return t.new_empty(shape, dtype=_t.float32)
    with _t.on_stream(other):
        return t.new_empty(shape, dtype=_t.float32)


def _like(t, other):
    """A new tensor like t, which is contiguous."""
    if other is None:
        return _t.empty_like(t)
    with _t.on_stream(other):
        return _t.empty_like(t)


def _workspace(workspace, need, t, other):
    """The caller's workspace, or a new one on t's device (of t's type, whose creation costs the least)."""
    if workspace is None:
        return _new(t, (need // t.element_size() + 1,), other)
    dev = t.get_device()
    if workspace.dtype != _t.uint8 or workspace.get_device() != dev or not workspace.is_contiguous() or \
            workspace.numel() < need:
        raise ValueError("workspace must be a contiguous uint8 tensor of at least %d bytes on GPU %d" % (need, dev))
    return workspace


class FfnPlan:
    """Owns an ffn plan: Y = (act(X Wg^T) * (X Wu^T)) Wo^T for X [N, d_in]."""

    def __init__(self, d_in: int, d_ff: int, d_out: int | None = None, dtype: str = "fp32", activation: str = "silu"):
        self.d_in, self.d_ff = int(d_in), int(d_ff)
        self.d_out = self.d_in if d_out is None else int(d_out)
        self.dtype, self.activation = dtype, activation
        _code(_DTYPES, dtype, "dtype")
        self._h = ffn_plan(self.d_in, self.d_ff, self.d_out, activation, dtype)
        self._tdt = _t.dtypes[dtype]

    def forward(self, x, w_in, w_out, save=False, out=None, saved=None, workspace=None, stream=None):
        """x: [N, d_in], rows may be strided; w_in: [2 d_ff, d_in], the gate's rows, then the up projection's;
        w_out: [d_out, d_ff].  Returns [N, d_out]; with save=True (or `saved`, a [N, 2 d_ff] fp32 tensor to write)
        also the values that backward() reads."""
        tdt, di, df, do = self._tdt, self.d_in, self.d_ff, self.d_out
        ldx = _rows(x, tdt, None, di, "x")
        N, dev = x.shape[0], x.get_device()
        wi, wo = _whole(w_in, tdt, (2 * df, di), "w_in", dev), _whole(w_out, tdt, (do, df), "w_out", dev)
        sp, other = _stream(stream, dev)
        if out is None:
            out = _new(x, (N, do), other)
        if save and saved is None:
            saved = _new32(x, (N, 2 * df), other)
        need = ffn_workspace_bytes(self._h, N)
        ws = _workspace(workspace, need, x, other)
        _call("ffn_forward", self._h, x.data_ptr(), ldx, wi, wo, _whole(out, tdt, (N, do), "out", dev),
              _whole(saved, _t.float32, (N, 2 * df), "saved", dev), N, ws.data_ptr(), need, sp)
        return out if saved is None else (out, saved)

    def backward(self, x, w_in, w_out, saved, grad_out, need_x=True, need_w_in=True, need_w_out=True, workspace=None,
                 stream=None):
        """(grad_x, grad_w_in, grad_w_out) of sum(grad_out * forward(x, w_in, w_out)); one not asked for is None.
        saved: what forward() returned beside Y; x and grad_out may have strided rows."""
        tdt, di, df, do = self._tdt, self.d_in, self.d_ff, self.d_out
        ldx = _rows(x, tdt, None, di, "x")
        N, dev = x.shape[0], x.get_device()
        ldg = _rows(grad_out, tdt, N, do, "grad_out", dev)
        wi, wo = _whole(w_in, tdt, (2 * df, di), "w_in", dev), _whole(w_out, tdt, (do, df), "w_out", dev)
        sv = _whole(saved, _t.float32, (N, 2 * df), "saved", dev)
        if not (need_x or need_w_in or need_w_out):
            return None, None, None
        sp, other = _stream(stream, dev)
        gx = _new(x, (N, di), other) if need_x else None
        gwi = _like(w_in, other) if need_w_in else None
        gwo = _like(w_out, other) if need_w_out else None
        need = ffn_backward_workspace_bytes(self._h, N)
        ws = _workspace(workspace, need, x, other)
        ptr = lambda t: t.data_ptr() if t is not None else None
        _call("ffn_backward", self._h, x.data_ptr(), ldx, wi, wo, sv, grad_out.data_ptr(), ldg, ptr(gx), ptr(gwi), ptr(gwo),
              N, ws.data_ptr(), need, sp)
        return gx, gwi, gwo

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            ffn_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class NormPlan:
    """The norms before and after a block: N(v; w) = v / sqrt(mean(v^2) + eps) * w over rows of `width` values.

    rows_per_gate consecutive rows share one row of the gate; `dropout` is the probability of dropping a value of
    the block's normed output."""

    def __init__(self, width: int, dtype: str = "fp32", eps: float = 1e-6, rows_per_gate: int = 1,
                 dropout: float = 0.0):
        self.width, self.dtype, self.eps = int(width), dtype, float(eps)
        self.rows_per_gate, self.dropout = int(rows_per_gate), float(dropout)
        self._code = _code(_DTYPES, dtype, "dtype")
        self._tdt = _t.dtypes[dtype]
        self._plain = self._describe(0, 0)
        if ffn_norm_workspace_bytes(self._plain, 0, 0) < 0:
            raise ValueError("width must be 1 .. %d, eps positive, rows_per_gate at least 1 and dropout within [0, 1]"
                             % FFN_MAX_WIDTH)

    def _norm(self, seed=0, offset=0):
        if self.dropout == 0.0:   # the generator is not asked
            return self._plain
        return self._describe(seed, offset)

    def _describe(self, seed, offset):
        return ffn_norm(self.width, self.rows_per_gate, self._code, self.eps, self.dropout, _word(seed), _word(offset))

    def forward(self, x, w=None, out=None, rstd=None, stream=None):
        """(u, rstd): u = N(x; w) for x [N, width], rows may be strided, and the rows' 1 / sqrt(mean + eps)."""
        tdt, D = self._tdt, self.width
        ldx = _rows(x, tdt, None, D, "x")
        N, dev = x.shape[0], x.get_device()
        wp = _whole(w, tdt, (D,), "w", dev)
        sp, other = _stream(stream, dev)
        if out is None:
            out, ldu = _new(x, (N, D), other), D
        else:
            ldu = _rows(out, tdt, N, D, "out", dev)
        if rstd is None:
            rstd = _new32(x, (N,), other)
        _call("ffn_norm_forward", self._plain, x.data_ptr(), ldx, wp, out.data_ptr(), ldu,
              _whole(rstd, _t.float32, (N,), "rstd", dev), N, sp)
        return out, rstd

    def backward(self, x, w, rstd, grad_out, need_x=True, need_w=True, workspace=None, stream=None):
        """(grad_x, grad_w) of sum(grad_out * N(x; w)); one not asked for is None."""
        tdt, D = self._tdt, self.width
        ldx = _rows(x, tdt, None, D, "x")
        N, dev = x.shape[0], x.get_device()
        ldg = _rows(grad_out, tdt, N, D, "grad_out", dev)
        wp, rp = _whole(w, tdt, (D,), "w", dev), _whole(rstd, _t.float32, (N,), "rstd", dev)
        if not (need_x or need_w):
            return None, None
        sp, other = _stream(stream, dev)
        norm = self._plain
        gx = _new(x, (N, D), other) if need_x else None
        gw = _new(x, (D,), other) if need_w else None
        need = ffn_norm_workspace_bytes(norm, N, 0)
        ws = _workspace(workspace, need, x, other)
        _call("ffn_norm_backward", norm, x.data_ptr(), ldx, wp, rp, grad_out.data_ptr(), ldg,
              gx.data_ptr() if need_x else None, gw.data_ptr() if need_w else None, N, ws.data_ptr(), need, sp)
        return gx, gw

    def _gates(self, N):
        return -(-N // self.rows_per_gate)

    def residual(self, x, h, w=None, gate=None, scale=None, w_next=None, next_norm=True, seed=0, offset=0, out=None,
                 stream=None):
        """(y, u, stats): y = x + scale * gate * drop(N(h; w)) and u = N(y; w_next) (None with next_norm=False).

        x, h: [N, width]; gate: [ceil(N / rows_per_gate), width]; scale, w, w_next: [width]; each of the four may be
        None (ones).  seed and offset choose the dropout's draws (see dropout()).  stats [2, N] holds the
        1 / sqrt(mean + eps) of h's and of y's rows, for residual_backward().  out may be x."""
        tdt, D = self._tdt, self.width
        if not x.is_cuda or x.dim() != 2:
            raise ValueError("x must be a %s CUDA tensor [N, %d]" % (tdt, D))
        N, dev = x.shape[0], x.get_device()
        xp, hp = _whole(x, tdt, (N, D), "x", dev), _whole(h, tdt, (N, D), "h", dev)
        wp, sc = _whole(w, tdt, (D,), "w", dev), _whole(scale, tdt, (D,), "scale", dev)
        gp, np_ = _whole(gate, tdt, (self._gates(N), D), "gate", dev), _whole(w_next, tdt, (D,), "w_next", dev)
        sp, other = _stream(stream, dev)
        if out is None:
            out = _like(h, other)
        u = _like(h, other) if next_norm else None
        stats = _new32(x, (2, N), other)
        _call("ffn_residual_forward", self._norm(seed, offset), xp, hp, wp, gp, sc, np_, _whole(out, tdt, (N, D), "out", dev),
                             u.data_ptr() if next_norm else None, stats.data_ptr(), N, sp)
        return out, u, stats

    def residual_backward(self, h, y, w, stats, grad_y, grad_u, gate=None, scale=None, w_next=None, seed=0, offset=0,
                          workspace=None, stream=None):
        """(grad_x, grad_h, grad_w, grad_gate, grad_scale, grad_w_next) of sum(grad_y * y) + sum(grad_u * u) for
        residual() with the same arguments; those of arguments that are None are None.  grad_y or grad_u may be
        None (zero), not both."""
        tdt, D = self._tdt, self.width
        if not h.is_cuda or h.dim() != 2:
            raise ValueError("h must be a %s CUDA tensor [N, %d]" % (tdt, D))
        if grad_y is None and grad_u is None:
            raise ValueError("one of grad_y and grad_u must be given")
        N, dev = h.shape[0], h.get_device()
        hp, yp = _whole(h, tdt, (N, D), "h", dev), _whole(y, tdt, (N, D), "y", dev)
        wp, sc = _whole(w, tdt, (D,), "w", dev), _whole(scale, tdt, (D,), "scale", dev)
        gp, np_ = _whole(gate, tdt, (self._gates(N), D), "gate", dev), _whole(w_next, tdt, (D,), "w_next", dev)
        st = _whole(stats, _t.float32, (2, N), "stats", dev)
        gyp, gup = _whole(grad_y, tdt, (N, D), "grad_y", dev), _whole(grad_u, tdt, (N, D), "grad_u", dev)
        sp, other = _stream(stream, dev)
        gx, gh = _like(h, other), _like(h, other)
        gw, gs, gn, gg = (None if t is None else _like(t, other) for t in (w, scale, w_next, gate))
        norm = self._norm(seed, offset)
        need = ffn_norm_workspace_bytes(norm, N, 1)
        ws = _workspace(workspace, need, h, other)
        ptr = lambda t: t.data_ptr() if t is not None else None
        _call("ffn_residual_backward", norm, hp, yp, wp, gp, sc, np_, st, gyp, gup, gx.data_ptr(), gh.data_ptr(), ptr(gw),
              ptr(gg), ptr(gs), ptr(gn), N, ws.data_ptr(), need, sp)
        return gx, gh, gw, gg, gs, gn


def dropout(x, p: float, seed: int, offset: int = 0, out=None, stream=None):
    """Dropout of x [..., width] by a counter-based generator: the values kept, scaled by 1 / (1 - p) with p rounded
    to a multiple of 2^-16.  Which are kept depends on (seed, offset, row, column) alone, with the leading dimensions
    flattened to rows; the gradient is the same call on the gradient.  x: contiguous, or [N, width] with strided
    rows; out may be x."""
    code = _t.codes.get(x.dtype)
    if code is None or not x.is_cuda or x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be an fp32, bf16 or fp16 CUDA tensor [..., width]")
    width, dev = x.shape[-1], x.get_device()
    N = x.numel() // width
    if x.is_contiguous():
        ldx = width
    elif x.dim() == 2:
        ldx = _rows(x, x.dtype, N, width, "x")
    else:
        raise ValueError("x must be contiguous, or [N, width] with strided rows")
    sp, other = _stream(stream, dev)
    if out is None:
        out, ldy = _like(x, other) if ldx == width else _new(x, x.shape, other), width
    elif out.shape != x.shape or out.get_device() != dev or out.dtype != x.dtype:
        raise ValueError("out must have the shape, type and device of x")
    elif out.is_contiguous():
        ldy = width
    elif out.dim() == 2:
        ldy = _rows(out, x.dtype, N, width, "out", dev)
    else:
        raise ValueError("out must be contiguous, or [N, width] with strided rows")
    _call("ffn_dropout", x.data_ptr(), ldx, out.data_ptr(), ldy, N, width, code, float(p), _word(seed), _word(offset), sp)
    return out
