"""Binding of include/experts.h: rows sorted by expert and brought back with
weights, and the experts' gated feed-forward blocks.

As in the package itself: the functions carry the C names and take device
pointers and a HIP stream; ``Routes`` takes and returns CUDA (HIP) torch tensors.
Outputs and workspaces that the caller does not give are allocated here, for the
stream that uses them.
"""
from __future__ import annotations

import ctypes

from ._ffn import _call, _code, _DTYPES, _entry, _new, _new32, _rows, _stream, _t, _whole

FFN_MAX_EXPERTS = 1024
__all__ = ["FFN_MAX_EXPERTS", "ffn_route", "ffn_route_workspace_bytes", "ffn_route_gather", "ffn_route_combine",
           "ffn_route_combine_backward", "Routes"]

_i32, _i64, _vp, _int = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
SIGNATURES = {
    "ffn_route": (_int, [_vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _i64, _vp]),
    "ffn_route_workspace_bytes": (_i64, [_i64, _i32, _i32]),
    "ffn_route_gather": (_int, [_vp, _i64, _vp, _vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp]),
    "ffn_route_combine": (_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i32, _i64, _i32, _vp]),
    "ffn_route_combine_backward": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp]),
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

    All three are int32 tensors on the GPU; nothing is copied to the host."""

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


def _new_int(t, shape, other):
    if other is None:
        return t.new_empty(shape, dtype=_t.int32)
    with _t.on_stream(other):
        return t.new_empty(shape, dtype=_t.int32)
