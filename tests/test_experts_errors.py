"""Refusals of include/experts.h and of the layer norm that the host decides before any HIP call, without a GPU."""
import ctypes

import pytest

import paper_2602_21466_amd as lib

E, U, D = lib.CGTP_EINVAL, lib.CGTP_EUNSUP, lib.CGTP_EDTYPE


@pytest.fixture
def p():
    buf = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(buf) + 255) & ~255


@pytest.mark.parametrize("kw", [{"width": 0}, {"width": (1 << 20) + 1}, {"eps": 0.0}, {"eps": float("nan")}, {"eps": float("inf")}])
def test_layer_descriptions(kw):
    with pytest.raises(ValueError):
        lib.LayerNormPlan(**dict({"width": 8}, **kw))
    n = lib.ffn_norm(8, 1, 0, 1e-6, 0.0, 0, 0)
    for k, v in kw.items():
        setattr(n, k, v)
    assert lib.ffn_layer_workspace_bytes(n, 4) == -1


@pytest.mark.parametrize("width", [1, 7, 64, 300, 1401, 5001, 20001, 1 << 20])
def test_layer_workspace_of_any_rows(width):
    for dtype in (0, 2, 3):
        n = lib.ffn_norm(width, 1, dtype, 1e-6, 0.0, 0, 0)
        for rows in (0, 1, 5, 255, 256, 4097, 100000, 1 << 30):
            assert lib.ffn_layer_workspace_bytes(n, rows) >= 0
        assert lib.ffn_layer_workspace_bytes(n, -1) == -1 and lib.ffn_layer_workspace_bytes(n, (1 << 30) + 1) == -1


def test_layer_refusals(p):
    f = lib._load()
    n = lib.ffn_norm(8, 1, 0, 1e-6, 0.0, 0, 0)
    call = lambda n=n, x=p, ldx=8, w=p + 1024, b=p + 2048, u=p + 4096, ldu=8, st=p + 8192, N=4: \
        f.ffn_layer_forward(n, x, ldx, w, b, u, ldu, st, N, None)
    assert call(n=None) == E and call(N=-1) == E and call(ldx=7) == E and call(ldu=7) == E and call(x=None) == E
    assert call(u=None) == E and call(u=p + 32) == E and call(u=p + 1040) == E and call(u=p + 2050) == E and call(st=p) == E
    assert call(x=p + 1) == E and call(st=p + 8194) == E and call(ldx=1 << 22) == U and call(N=(1 << 30) + 1) == U
    assert call(u=p, ldu=9) == E and call(N=0) == lib.CGTP_OK
    n.dtype = 1
    assert call() == D
    n.dtype = 0
    need = lib.ffn_layer_workspace_bytes(n, 4)
    back = lambda x=p, st=p + 1024, gu=p + 2048, gx=p + 4096, gw=p + 8192, gb=p + 8448, ws=p + 16384, size=need, N=4: \
        f.ffn_layer_backward(n, x, 8, None, st, gu, 8, gx, gw, gb, N, ws, size, None)
    assert back(x=None) == E and back(st=None) == E and back(gu=None) == E and back(gx=None, gw=None, gb=None) == E
    assert back(size=need - 1) == E and back(ws=None) == E and back(ws=p + 16384 + 4) == E and back(gx=p) == E
    assert back(gw=p + 8440) == E and back(gb=p + 8193) == E and back(ws=p + 4096) == E and back(N=-1) == E


def test_route_sizes():
    ws = lib.ffn_route_workspace_bytes
    assert ws(0, 1, 1) == 0 and ws(8192, 1, 4) == 0 and ws(8193, 1, 4) > 0 and ws(1 << 30, 1, 1024) % 256 == 0
    assert ws(-1, 1, 1) == -1 and ws(1, 0, 1) == -1 and ws(1, 1, 0) == -1
    assert ws(1, 1025, 1) == -1 and ws(1, 1, 1025) == -1 and ws((1 << 30) + 1, 1, 1) == -1 and ws(1 << 29, 3, 1) == -1


def test_route_refusals(p):
    f = lib._load()
    call = lambda index=p, size=8, N=4, k=2, e=3, place=p + 1024, source=p + 2048, off=p + 4096, ws=None, need=0: \
        f.ffn_route(index, size, N, k, e, place, source, off, ws, need, None)
    assert call(index=None) == E and call(place=None) == E and call(source=None) == E and call(off=None) == E
    assert call(size=2) == E and call(N=-1) == E and call(k=0) == E and call(e=0) == E and call(e=1025) == U
    assert call(k=1025) == U and call(N=1 << 30) == U and call(index=p + 4) == E and call(off=p + 4098) == E
    assert call(place=p + 8) == E and call(source=p + 1040) == E and call(off=p + 2052) == E
    assert call(N=10000, place=p + (1 << 20), source=p + (2 << 20), off=p + (3 << 20)) == E   # no workspace


def test_row_refusals(p):
    f = lib._load()
    a = dict(x=p, ldx=8, place=p + 4096, off=p + 4352, xs=p + 8192, N=4, k=2, e=3, width=8, dtype=0)
    g = lambda **kw: f.ffn_route_gather(*dict(a, **kw).values(), None)
    assert g(x=None) == E and g(place=None) == E and g(off=None) == E and g(xs=None) == E and g(ldx=7) == E
    assert g(N=-1) == E and g(width=0) == E and g(dtype=1) == D and g(width=1 << 21, ldx=1 << 21) == U and g(ldx=1 << 22) == U
    assert g(xs=p + 64) == E and g(xs=p + 4100) == E and g(x=p + 2) == E and g(k=0) == E and g(e=1025) == U
    assert g(N=0) == lib.CGTP_OK
    a2 = dict(ys=p, place=p + 4096, w=p + 4352, y=p + 8192, ldy=8, N=4, k=2, width=8, dtype=0)
    c = lambda **kw: f.ffn_route_combine(*dict(a2, **kw).values(), None)
    assert c(ys=None) == E and c(place=None) == E and c(y=None) == E and c(ldy=7) == E and c(dtype=7) == D
    assert c(y=p + 32) == E and c(y=p + 4352) == E and c(w=p + 4353) == E and c(N=0) == lib.CGTP_OK
    a3 = dict(ys=p, place=p + 4096, off=p + 4352, w=p + 4608, gy=p + 8192, ldg=8, gys=p + 16384, gw=p + 32768, N=4, k=2,
              e=3, width=8, dtype=0)
    b = lambda **kw: f.ffn_route_combine_backward(*dict(a3, **kw).values(), None)
    assert b(ys=None) == E and b(gys=None, gw=None) == E and b(gy=None) == E and b(ldg=7) == E and b(off=None) == E
    assert b(gys=p) == E and b(gw=p + 16384) == E and b(gw=p + 4608) == E and b(gw=p + 32769) == E and b(dtype=1) == D
    assert b(N=0) == lib.CGTP_OK


@pytest.mark.parametrize("args,rc", [((0, 4, 4, 4, 0, 2), E), ((4, 0, 4, 4, 0, 2), E), ((4, 4, 0, 4, 0, 2), E), ((4, 4, 4, -1, 0, 2), E),
                                     ((4, 4, 4, 4, 3, 2), E), ((4, 4, 4, 4, 0, 1), D), ((1025, 4, 4, 4, 0, 2), U),
                                     ((4, (1 << 20) + 1, 4, 4, 0, 2), U), ((1024, 4, 1 << 20, 4, 0, 2), U)])
def test_experts_plan_refusals(args, rc):
    h = ctypes.c_void_p()
    assert lib._load().ffn_experts_plan(*args, ctypes.byref(h)) == rc and h.value is None


def test_experts_null_arguments():
    f = lib._load()
    assert f.ffn_experts_plan(2, 4, 4, 4, 0, 0, None) == E and f.ffn_experts_destroy(None) == lib.CGTP_OK
    assert f.ffn_experts_workspace_bytes(None, 4, 1) == -1 and f.ffn_experts_backward_workspace_bytes(None, 4, 1) == -1
    assert f.ffn_experts_forward(None, None, 0, *[None] * 7, 1, 1, None, 0, None) == E
    assert f.ffn_experts_backward(None, None, 0, *[None] * 10, 1, 1, None, 0, None) == E
