"""Binding of include/experts.h: rows sorted by expert and brought back with
weights, and the experts' gated feed-forward blocks.

As in the package itself: the functions carry the C names and take device
pointers and a HIP stream; ``Routes`` and ``ExpertsPlan`` take and return CUDA (HIP)
torch tensors.  Outputs and workspaces that the caller does not give are allocated here, for the
stream that uses them.
"""
from __future__ import annotations

import ctypes

from ._ffn import _ACTIVATIONS, _call, _code, _DTYPES, _entry, _like, _new, _new32, _rows, _stream, _t, _whole, _workspace

FFN_MAX_EXPERTS = 1024
__all__ = ["FFN_MAX_EXPERTS", "ffn_route", "ffn_route_workspace_bytes", "ffn_route_gather", "ffn_route_combine",
           "ffn_route_combine_backward", "ffn_experts_plan", "ffn_experts_destroy", "ffn_experts_workspace_bytes",
           "ffn_experts_backward_workspace_bytes", "ffn_experts_forward", "ffn_experts_backward", "Routes", "ExpertsPlan"]

_i32, _i64, _vp, _int = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
SIGNATURES = {
    "ffn_route": (_int, [_vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _i64, _vp]),
    "ffn_route_workspace_bytes": (_i64, [_i64, _i32, _i32]),
    "ffn_route_gather": (_int, [_vp, _i64, _vp, _vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp]),
    "ffn_route_combine": (_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i32, _i64, _i32, _vp]),
    "ffn_route_combine_backward": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp]),
    "ffn_experts_plan": (_int, [_i32, _i64, _i64, _i64, _i32, _i32, ctypes.POINTER(_vp)]),
    "ffn_experts_destroy": (_int, [_vp]),
    "ffn_experts_workspace_bytes": (_i64, [_vp, _i64, _i32]),
    "ffn_experts_backward_workspace_bytes": (_i64, [_vp, _i64, _i32]),
    "ffn_experts_forward": (_int, [_vp, _vp, _i64] + [_vp] * 7 + [_i64, _i32, _vp, _i64, _vp]),
    "ffn_experts_backward": (_int, [_vp, _vp, _i64] + [_vp] * 10 + [_i64, _i32, _vp, _i64, _vp]),
}


# ---------------------------------------------------------------- C names

def ffn_route(index_ptr, index_bytes, N, per_row, experts, place_ptr, source_ptr, offsets_ptr, ws_ptr, ws_bytes,
              stream_ptr=None) -> None:
    _call("ffn_route", index_ptr, index_bytes, N, per_row, experts, place_ptr, source_ptr, offsets_ptr, ws_ptr, ws_bytes,
          stream_ptr)


def ffn_route_workspace_bytes(N: int, per_row: int, experts: int) -> int:
    return _entry("ffn_route_workspace_bytes")(N, per_row, experts)


def ffn_route_gather(x_ptr, ldx, place_ptr, offsets_ptr, xs_ptr, N, per_row, experts, width, dtype,
                     stream_ptr=None) -> None:
    _call("ffn_route_gather", x_ptr, ldx, place_ptr, offsets_ptr, xs_ptr, N, per_row, experts, width,
          _code(_DTYPES, dtype, "dtype"), stream_ptr)


def ffn_route_combine(ys_ptr, place_ptr, weights_ptr, y_ptr, ldy, N, per_row, width, dtype, stream_ptr=None) -> None:
    _call("ffn_route_combine", ys_ptr, place_ptr, weights_ptr, y_ptr, ldy, N, per_row, width,
          _code(_DTYPES, dtype, "dtype"), stream_ptr)


def ffn_route_combine_backward(ys_ptr, place_ptr, offsets_ptr, weights_ptr, gy_ptr, ldg, gys_ptr, gw_ptr, N, per_row,
                               experts, width, dtype, stream_ptr=None) -> None:
    _call("ffn_route_combine_backward", ys_ptr, place_ptr, offsets_ptr, weights_ptr, gy_ptr, ldg, gys_ptr, gw_ptr, N,
          per_row, experts, width, _code(_DTYPES, dtype, "dtype"), stream_ptr)


def ffn_experts_plan(experts: int, d_in: int, d_ff: int, d_out: int, activation="silu", dtype="fp32") -> ctypes.c_void_p:
    h = ctypes.c_void_p()
    _call("ffn_experts_plan", int(experts), int(d_in), int(d_ff), int(d_out), _code(_ACTIVATIONS, activation, "activation"),
          _code(_DTYPES, dtype, "dtype"), ctypes.byref(h))
    return h


def ffn_experts_destroy(plan) -> None:
    _call("ffn_experts_destroy", plan)


def ffn_experts_workspace_bytes(plan, N: int, per_row: int) -> int:
    return _entry("ffn_experts_workspace_bytes")(plan, N, per_row)


def ffn_experts_backward_workspace_bytes(plan, N: int, per_row: int) -> int:
    return _entry("ffn_experts_backward_workspace_bytes")(plan, N, per_row)


def ffn_experts_forward(plan, x_ptr, ldx, place_ptr, source_ptr, offsets_ptr, w_in_ptr, w_out_ptr, y_ptr, saved_ptr, N,
                        per_row, ws_ptr, ws_bytes, stream_ptr=None) -> None:
    _call("ffn_experts_forward", plan, x_ptr, ldx, place_ptr, source_ptr, offsets_ptr, w_in_ptr, w_out_ptr, y_ptr,
          saved_ptr, N, per_row, ws_ptr, ws_bytes, stream_ptr)


def ffn_experts_backward(plan, x_ptr, ldx, place_ptr, source_ptr, offsets_ptr, w_in_ptr, w_out_ptr, saved_ptr, gy_ptr,
                         gx_ptr, gw_in_ptr, gw_out_ptr, N, per_row, ws_ptr, ws_bytes, stream_ptr=None) -> None:
    _call("ffn_experts_backward", plan, x_ptr, ldx, place_ptr, source_ptr, offsets_ptr, w_in_ptr, w_out_ptr, saved_ptr,
          gy_ptr, gx_ptr, gw_in_ptr, gw_out_ptr, N, per_row, ws_ptr, ws_bytes, stream_ptr)


# ---------------------------------------------------------------- convenience

def _width(t, what):
    """The type's code and the width of t, a CUDA tensor [rows, width] of a type that the calls take."""
    if not t.is_cuda or t.dim() != 2 or t.shape[1] < 1:
        raise ValueError("%s must be a CUDA tensor [rows, width]" % what)
    code = _t.codes.get(t.dtype)
    if code is None:
        raise ValueError("%s must be fp32, bf16 or fp16" % what)
    return code, t.shape[1]


class Routes:
    """Rows sorted by expert: the order, and the way there and back.

    index: [N, per_row] (or [N]: one choice a row), int32 or int64, contiguous: the experts that each row chose; a
    value outside 0 .. experts - 1 (-1, say) chooses none.  Rows go to S = N * per_row sorted rows, expert by expert,
    those of an expert in the order of the rows:

        offsets [experts + 1]  expert e has the sorted rows offsets[e] .. offsets[e + 1] - 1
        place (like index)     the sorted row of each choice, -1 where it chose none
        source [S]             the choice n * per_row + k of each sorted row, -1 from offsets[experts] on

    All three are int32 tensors on the GPU; nothing is copied to the host.  They are memory of the stream that they were
    made on: where another uses them, keep them until it is done."""

    def __init__(self, index, experts: int, stream=None):
        if not index.is_cuda or index.dim() not in (1, 2) or not index.is_contiguous() or \
                index.dtype not in (_t.int32, _t.int64) or (index.dim() == 2 and index.shape[1] < 1):
            raise ValueError("index must be a contiguous int32 or int64 CUDA tensor [N, per_row] or [N]")
        self.experts, self.rows = int(experts), index.shape[0]
        self.per_row = 1 if index.dim() == 1 else index.shape[1]
        need = ffn_route_workspace_bytes(self.rows, self.per_row, self.experts)
        if need < 0:
            raise ValueError("experts and choices a row must be 1 .. %d, all choices 2^30 or fewer" % FFN_MAX_EXPERTS)
        self.device = index.get_device()
        sp, other = _stream(stream, self.device)
        i32 = _t.int32
        self.place = _new_int(index, index.shape, other)
        self.source = _new_int(index, (index.numel(),), other)
        self.offsets = _new_int(index, (self.experts + 1,), other)
        ws = _new_int(index, (need // 4,), other) if need else None
        _call("ffn_route", index.data_ptr(), 4 if index.dtype == i32 else 8, self.rows, self.per_row, self.experts,
              self.place.data_ptr(), self.source.data_ptr(), self.offsets.data_ptr(), ws.data_ptr() if need else None,
              need, sp)

    def _weights(self, weights):
        return _whole(weights, _t.float32, self.place.shape, "weights", self.device)

    def _sorted(self, t, dtype, width, what):
        return _whole(t, dtype, (self.source.shape[0], width), what, self.device)

    def gather(self, x, out=None, stream=None):
        """xs [S, width]: the rows of x [N, width] (rows may be strided) in the sorted order; zeros behind the last."""
        code, D = _width(x, "x")
        ldx = _rows(x, x.dtype, self.rows, D, "x", self.device)
        sp, other = _stream(stream, self.device)
        if out is None:
            out = _new(x, (self.source.shape[0], D), other)
        _call("ffn_route_gather", x.data_ptr(), ldx, self.place.data_ptr(), self.offsets.data_ptr(),
              self._sorted(out, x.dtype, D, "out"), self.rows, self.per_row, self.experts, D, code, sp)
        return out

    def gather_backward(self, grad_out, out=None, stream=None):
        """The gradient [N, width] of sum(grad_out * gather(x)) with respect to x; grad_out [S, width]."""
        return self.combine(grad_out, None, out, stream)

    def combine(self, ys, weights=None, out=None, stream=None):
        """y [N, width], y[n] = sum over k of weights[n, k] * ys[place[n, k]], for ys [S, width] in the sorted order and
        weights like index, 32-bit floats (None: ones).  Choices of no expert add nothing."""
        code, D = _width(ys, "ys")
        yp, wp = self._sorted(ys, ys.dtype, D, "ys"), self._weights(weights)
        sp, other = _stream(stream, self.device)
        if out is None:
            out, ldy = _new(ys, (self.rows, D), other), D
        else:
            ldy = _rows(out, ys.dtype, self.rows, D, "out", self.device)
        _call("ffn_route_combine", yp, self.place.data_ptr(), wp, out.data_ptr(), ldy, self.rows, self.per_row, D, code, sp)
        return out

    def combine_backward(self, ys, weights, grad_out, need_ys=True, need_weights=True, stream=None):
        """(grad_ys, grad_weights) of sum(grad_out * combine(ys, weights)), grad_out [N, width] (rows may be strided);
        one not asked for is None (ys is then not read for grad_ys, nor weights for grad_weights, and may be None).
        grad_ys is zero behind the last sorted row, grad_weights where no expert was chosen."""
        code, D = _width(grad_out, "grad_out")
        ldg = _rows(grad_out, grad_out.dtype, self.rows, D, "grad_out", self.device)
        if need_weights and ys is None:
            raise ValueError("grad_weights needs ys")
        yp = self._sorted(ys, grad_out.dtype, D, "ys") if need_weights else None
        wp = self._weights(weights) if need_ys else None
        if not (need_ys or need_weights):
            return None, None
        sp, other = _stream(stream, self.device)
        gys = _new(grad_out, (self.source.shape[0], D), other) if need_ys else None
        gw = _new32(grad_out, self.place.shape, other) if need_weights else None
        _call("ffn_route_combine_backward", yp, self.place.data_ptr(), self.offsets.data_ptr(), wp, grad_out.data_ptr(), ldg,
              gys.data_ptr() if need_ys else None, gw.data_ptr() if need_weights else None, self.rows, self.per_row,
              self.experts, D, code, sp)
        return gys, gw


class ExpertsPlan:
    """Owns a plan of `experts` gated blocks of one shape: Y_p = (act(X_p Wg_e^T) * (X_p Wu_e^T)) Wo_e^T for the sorted
    rows p of each expert e, in the order that a Routes of as many experts holds."""

    def __init__(self, experts: int, d_in: int, d_ff: int, d_out: int | None = None, dtype: str = "fp32",
                 activation: str = "silu"):
        self.experts, self.d_in, self.d_ff = int(experts), int(d_in), int(d_ff)
        self.d_out = self.d_in if d_out is None else int(d_out)
        self.dtype, self.activation = dtype, activation
        _code(_DTYPES, dtype, "dtype")
        self._h = ffn_experts_plan(self.experts, self.d_in, self.d_ff, self.d_out, activation, dtype)
        self._tdt = _t.dtypes[dtype]

    def _args(self, x, routes, w_in, w_out):
        if not isinstance(routes, Routes) or routes.experts != self.experts:
            raise ValueError("routes must be a Routes of %d experts" % self.experts)
        dev = routes.device
        ldx = _rows(x, self._tdt, routes.rows, self.d_in, "x", dev)
        return dev, ldx, _whole(w_in, self._tdt, (self.experts, 2 * self.d_ff, self.d_in), "w_in", dev), \
            _whole(w_out, self._tdt, (self.experts, self.d_out, self.d_ff), "w_out", dev)

    def forward(self, x, routes, w_in, w_out, save=False, out=None, saved=None, workspace=None, stream=None):
        """x: [N, d_in], rows may be strided, N and the choices as in routes; w_in: [experts, 2 d_ff, d_in], of each
        expert the gate's rows, then the up projection's; w_out: [experts, d_out, d_ff].  Returns [S, d_out] in the
        sorted order, for Routes.combine(); rows from routes.offsets[experts] on are not written.  With save=True (or
        `saved`, a [S, 2 d_ff] fp32 tensor to write) also the values that backward() reads."""
        dev, ldx, wi, wo = self._args(x, routes, w_in, w_out)
        S, df, do = routes.source.shape[0], self.d_ff, self.d_out
        sp, other = _stream(stream, dev)
        if out is None:
            out = _new(x, (S, do), other)
        if save and saved is None:
            saved = _new32(x, (S, 2 * df), other)
        need = ffn_experts_workspace_bytes(self._h, routes.rows, routes.per_row)
        ws = _workspace(workspace, need, x, other)
        _call("ffn_experts_forward", self._h, x.data_ptr(), ldx, routes.place.data_ptr(), routes.source.data_ptr(),
              routes.offsets.data_ptr(), wi, wo, _whole(out, self._tdt, (S, do), "out", dev),
              _whole(saved, _t.float32, (S, 2 * df), "saved", dev), routes.rows, routes.per_row, ws.data_ptr(), need, sp)
        return out if saved is None else (out, saved)

    def backward(self, x, routes, w_in, w_out, saved, grad_out, need_x=True, need_w_in=True, need_w_out=True,
                 workspace=None, stream=None):
        """(grad_x, grad_w_in, grad_w_out) of sum(grad_out * forward(x, ...)) over the sorted rows of an expert, grad_out
        [S, d_out] (as Routes.combine_backward() gives it): grad_x [N, d_in] is the sum over a row's choices; one not
        asked for is None.  saved: what forward() returned beside Y."""
        dev, ldx, wi, wo = self._args(x, routes, w_in, w_out)
        S = routes.source.shape[0]
        gy = _whole(grad_out, self._tdt, (S, self.d_out), "grad_out", dev)
        sv = _whole(saved, _t.float32, (S, 2 * self.d_ff), "saved", dev)
        if not (need_x or need_w_in or need_w_out):
            return None, None, None
        sp, other = _stream(stream, dev)
        gx = _new(x, (routes.rows, self.d_in), other) if need_x else None
        gwi = _like(w_in, other) if need_w_in else None
        gwo = _like(w_out, other) if need_w_out else None
        need = ffn_experts_backward_workspace_bytes(self._h, routes.rows, routes.per_row)
        ws = _workspace(workspace, need, x, other)
        ptr = lambda t: t.data_ptr() if t is not None else None
        _call("ffn_experts_backward", self._h, x.data_ptr(), ldx, routes.place.data_ptr(), routes.source.data_ptr(),
              routes.offsets.data_ptr(), wi, wo, sv, gy, ptr(gx), ptr(gwi), ptr(gwo), routes.rows, routes.per_row,
              ws.data_ptr(), need, sp)
        return gx, gwi, gwo

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            ffn_experts_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _new_int(t, shape, other):
    if other is None:
        return t.new_empty(shape, dtype=_t.int32)
    with _t.on_stream(other):
        return t.new_empty(shape, dtype=_t.int32)
