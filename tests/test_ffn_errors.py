"""Refusals of include/ffn.h that the host decides before any HIP call, and the published definition that the
dropout's generator follows, without a GPU."""
import ctypes

import pytest

import paper_2602_21466_amd as lib


def _plan(*args):
    h = ctypes.c_void_p()
    return lib._load().ffn_plan(*args, ctypes.byref(h)), h.value


@pytest.mark.parametrize("args,rc", [((0, 4, 4, 0, 2), lib.CGTP_EINVAL), ((4, 0, 4, 0, 2), lib.CGTP_EINVAL),
                                     ((4, 4, -1, 0, 2), lib.CGTP_EINVAL), ((4, 4, 4, 3, 2), lib.CGTP_EINVAL),
                                     ((4, 4, 4, -1, 2), lib.CGTP_EINVAL), ((4, 4, 4, 0, 1), lib.CGTP_EDTYPE),
                                     ((4, 4, 4, 0, 9), lib.CGTP_EDTYPE), (((1 << 20) + 1, 4, 4, 0, 2), lib.CGTP_EUNSUP)])
def test_plan_refusals(args, rc):
    assert _plan(*args) == (rc, None)


def test_null_arguments():
    f = lib._load()
    assert f.ffn_plan(4, 4, 4, 0, 0, None) == lib.CGTP_EINVAL
    assert f.ffn_destroy(None) == lib.CGTP_OK
    assert f.ffn_workspace_bytes(None, 4) == -1 and f.ffn_backward_workspace_bytes(None, 4) == -1
    assert f.ffn_forward(None, None, 0, None, None, None, None, 1, None, 0, None) == lib.CGTP_EINVAL
    assert f.ffn_backward(None, None, 0, None, None, None, None, 0, None, None, None, 1, None, 0, None) == lib.CGTP_EINVAL
    assert f.ffn_norm_forward(None, None, 0, None, None, 0, None, 1, None) == lib.CGTP_EINVAL
    assert f.ffn_norm_workspace_bytes(None, 1, 0) == -1
    assert f.ffn_dropout(None, 4, None, 4, 2, 4, 0, 0.5, 1, 0, None) == lib.CGTP_EINVAL


@pytest.mark.parametrize("kw", [{"width": 0}, {"width": (1 << 20) + 1}, {"eps": 0.0}, {"eps": -1.0}, {"eps": float("nan")},
                                {"eps": float("inf")}, {"rows_per_gate": 0}, {"dropout": -0.1}, {"dropout": 1.5},
                                {"dropout": float("nan")}])
def test_norm_descriptions(kw):
    args = dict({"width": 8}, **kw)
    with pytest.raises(ValueError):
        lib.NormPlan(**args)
    n = lib.ffn_norm(8, 1, 0, 1e-6, 0.0, 0, 0)
    for k, v in kw.items():
        setattr(n, k, v)
    assert lib.ffn_norm_workspace_bytes(n, 4, 0) == -1


@pytest.mark.parametrize("width", [1, 7, 64, 300, 1401, 5001, 20001, 1 << 20])
@pytest.mark.parametrize("rows_per_gate", [1, 3, 1000, 1 << 30])
def test_norm_workspace_of_any_rows(width, rows_per_gate):
    for dtype in (0, 2, 3):
        n = lib.ffn_norm(width, rows_per_gate, dtype, 1e-6, 0.0, 0, 0)
        for rows in (0, 1, 5, 255, 256, 4097, 100000, 1 << 30):
            assert all(lib.ffn_norm_workspace_bytes(n, rows, r) >= 0 for r in (0, 1))


def test_norm_workspace_and_dtype():
    n = lib.ffn_norm(64, 1, 2, 1e-6, 0.0, 0, 0)
    assert lib.ffn_norm_workspace_bytes(n, 0, 0) >= 0
    assert lib.ffn_norm_workspace_bytes(n, 100, 1) % 256 == 0
    assert lib.ffn_norm_workspace_bytes(n, -1, 0) == -1 and lib.ffn_norm_workspace_bytes(n, 1, 2) == -1
    n.dtype = 1
    assert lib.ffn_norm_workspace_bytes(n, 1, 0) == -1
    with pytest.raises(ValueError):
        lib.NormPlan(8, dtype="fp64")


def test_dropout_refusals():
    f = lib._load()
    buf = ctypes.create_string_buffer(4096)
    p = ctypes.addressof(buf)
    call = lambda x=p, ldx=8, y=p + 2048, ldy=8, N=4, w=8, dt=0, q=0.5: f.ffn_dropout(x, ldx, y, ldy, N, w, dt, q, 1, 0, None)
    assert call(dt=1) == lib.CGTP_EDTYPE and call(N=-1) == lib.CGTP_EINVAL and call(w=0) == lib.CGTP_EINVAL
    assert call(q=1.5) == lib.CGTP_EINVAL and call(q=float("nan")) == lib.CGTP_EINVAL and call(ldx=7) == lib.CGTP_EINVAL
    assert call(x=p + 1) == lib.CGTP_EINVAL and call(y=p + 16) == lib.CGTP_EINVAL and call(y=p, ldy=9) == lib.CGTP_EINVAL
    assert call(N=(1 << 30) + 1) == lib.CGTP_EUNSUP and call(w=1 << 35, ldx=1 << 35, ldy=1 << 35, N=1) == lib.CGTP_EUNSUP
    assert call(N=0) == lib.CGTP_OK


def test_generator_against_published_values():
    """The generator's definition as the tests state it, against the known answers published with the method."""
    from test_ffn_gpu import _philox
    ones = 0xFFFFFFFF
    assert _philox((0,) * 4, (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert _philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert _philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
