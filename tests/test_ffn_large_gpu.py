"""The feed-forward sublayer where its kernels change form: large and ragged tiles, k in parts, wide rows, offsets past
32 bits; and the example that runs the operators together.  References in 64 bits on the GPU; tolerances as in
test_ffn_gpu.py, with 32-bit sums of up to 16384 terms (2^-24 sqrt(16384), 8e-6, for the longest)."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROUND = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}   # unit roundoff


def _setup():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_21466_amd as lib
    return torch, lib


def _dt(torch, dtype):
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]


def _rel(got, want):
    assert got.shape == want.shape and bool(got.isfinite().all())
    return float((got.double() - want).norm() / want.norm())


def _tol(dtype, roundings):
    return roundings * ROUND[dtype] + 8e-6


# rows, d_in, d_ff, d_out: whole 256-wide tiles; ragged ones; few tiles and long sums (k in parts, each epilogue); few
# rows in every form of theirs; rows of a tile that are one matrix's last
SIZES = [(2048, 512, 1024, 512), (1537, 776, 1000, 520), (130, 4100, 260, 8200), (260, 66, 8196, 70), (8192, 40, 36, 130),
         (24, 2048, 4096, 1024), (50, 1030, 2050, 514), (64, 300, 17000, 5), (9, 6000, 520, 1001), (5, 3, 9000, 4100),
         (700, 129, 2100, 1700), (16, 4096, 16384, 32)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,di,df,do", SIZES)
def test_block(N, di, df, do, dtype):
    torch, lib = _setup()
    g = torch.Generator(device="cuda").manual_seed(N)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda", dtype=torch.float64) * s[-1] ** -0.5).to(_dt(torch, dtype))
    x, wi, wo, gy = r(N, di) * di ** 0.5, r(2 * df, di), r(do, df), r(N, do)
    plan = lib.FfnPlan(di, df, do, dtype=dtype, activation="gelu")
    y, saved = plan.forward(x, wi, wo, save=True)
    grads = plan.backward(x, wi, wo, saved, gy)
    leaves = [t.double().requires_grad_(True) for t in (x, wi, wo)]
    z = leaves[0] @ leaves[1].T
    want = (z[:, :df] * torch.special.ndtr(z[:, :df]) * z[:, df:]) @ leaves[2].T
    want_g = torch.autograd.grad(want, leaves, gy.double())
    assert _rel(saved, z.detach()) <= 8e-6
    assert _rel(y, want.detach()) <= _tol(dtype, 2)     # H and the output
    for got, w in zip(grads, want_g):
        assert _rel(got, w) <= _tol(dtype, 2)           # dG and dU, or H, and the output
    again = plan.backward(x, wi, wo, saved, gy)         # no atomics: the same bits
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D,rpg", [(3, 40000, 2), (700, 8200, 90), (5000, 300, 1), (2500, 2048, 700), (40, 5, 3), (9000, 64, 4)])
def test_norms(N, D, rpg, dtype):
    torch, lib = _setup()
    g = torch.Generator(device="cuda").manual_seed(N + D)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64).to(_dt(torch, dtype))
    x, h, gy, gu, gate = r(N, D), r(N, D), r(N, D), r(N, D), r(-(-N // rpg), D)
    w, scale, wn = r(D), r(D), r(D)
    plan = lib.NormPlan(D, dtype=dtype, rows_per_gate=rpg, eps=1e-4)
    kw = {"gate": gate, "scale": scale, "w_next": wn}
    y, u, stats = plan.residual(x, h, w, **kw)
    grads = plan.residual_backward(h, y, w, stats, gy, gu, **kw)
    leaves = [t.double().requires_grad_(True) for t in (x, h, w, gate, scale, wn)]
    n = lambda v, c: v / (v.square().mean(1, keepdim=True) + 1e-4).sqrt() * c
    yr = leaves[0] + leaves[4] * leaves[3][torch.arange(N, device="cuda") // rpg] * n(leaves[1], leaves[2])
    ur = n(yr, leaves[5])
    want = torch.autograd.grad((yr, ur), leaves, (gy.double(), gu.double()))
    assert _rel(y, yr.detach()) <= _tol(dtype, 1) and _rel(u, ur.detach()) <= _tol(dtype, 1)
    for got, wt in zip(grads, want):
        assert _rel(got, wt) <= _tol(dtype, 3)          # y is read back rounded
    ub, rstd = plan.forward(x, w)
    gx, gw = plan.backward(x, w, rstd, gu)
    xr, wr = x.double().requires_grad_(True), w.double().requires_grad_(True)
    ref = n(xr, wr)
    want = torch.autograd.grad(ref, (xr, wr), gu.double())
    assert _rel(ub, ref.detach()) <= _tol(dtype, 1)
    assert _rel(gx, want[0]) <= _tol(dtype, 1) and _rel(gw, want[1]) <= _tol(dtype, 1)


def test_rows_past_32_bits():
    """Rows 2^21 elements apart: the last ones start past 2^31 elements and 2^32 bytes."""
    torch, lib = _setup()
    N, ld, d = 1100, 1 << 21, 64
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.empty(N, ld, dtype=torch.bfloat16, device="cuda")
    x = big[:, 8:8 + d]
    x.copy_(torch.randn(N, d, generator=g, device="cuda"))
    packed = x.contiguous()
    norm = lib.NormPlan(d, dtype="bf16")
    u, rstd = norm.forward(x)
    assert torch.equal(u, norm.forward(packed)[0])
    assert torch.equal(norm.backward(packed, None, rstd, x)[0], norm.backward(packed, None, rstd, packed)[0])
    assert torch.equal(lib.dropout(x, 0.5, seed=3), lib.dropout(packed, 0.5, seed=3))
    plan = lib.FfnPlan(d, 96, d, dtype="bf16")
    wi, wo = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((192, d), (d, 96)))
    y, saved = plan.forward(x, wi, wo, save=True)
    assert torch.equal(y, plan.forward(packed, wi, wo))
    for a, b in zip(plan.backward(x, wi, wo, saved, x), plan.backward(packed, wi, wo, saved, packed)):
        assert torch.equal(a, b)
    lib.dropout(packed, 0.5, seed=4, out=x)
    assert torch.equal(x, lib.dropout(packed, 0.5, seed=4))


def test_dropout_of_more_than_32_bits_of_values():
    torch, lib = _setup()
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    N, D = 70000, 65536
    x = torch.ones(N, D, dtype=torch.bfloat16, device="cuda")
    y = lib.dropout(x, 0.25, seed=11, out=x)
    # a row's draws do not depend on how many rows or columns the call has
    for row in (0, 32768, N - 1):
        part = torch.ones(row + 1, 24, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(y[row, :24], lib.dropout(part, 0.25, seed=11)[row])
    tail = (y[-64:] == 0).double().mean()
    assert abs(float(tail) - 0.25) <= 5 * np.sqrt(0.25 * 0.75 / (64 * D))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D,rpg", [(700, 5001, 100), (4500, 1401, 1), (1100, 1029, 64), (300, 2500, 1000), (6000, 77, 7)])
def test_residual_with_dropout(N, D, rpg, dtype):
    """Widths whose last eight columns two threads share, rows divided within and over gate rows: against the same
    formula in 64 bits with the mask that `dropout` gives, and in place of x."""
    torch, lib = _setup()
    g = torch.Generator(device="cuda").manual_seed(N + D)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64).to(_dt(torch, dtype))
    x, h, gy, gu, gate, w, scale, wn = r(N, D), r(N, D), r(N, D), r(N, D), r(-(-N // rpg), D), r(D), r(D), r(D)
    plan = lib.NormPlan(D, dtype=dtype, rows_per_gate=rpg, eps=1e-4, dropout=0.25)
    kw = {"gate": gate, "scale": scale, "w_next": wn, "seed": 77, "offset": 5}
    y, u, stats = plan.residual(x, h, w, **kw)
    grads = plan.residual_backward(h, y, w, stats, gy, gu, **kw)
    keep = (lib.dropout(torch.ones(N, D, device="cuda"), 0.25, seed=77, offset=5) != 0).double() / 0.75
    leaves = [t.double().requires_grad_(True) for t in (x, h, w, gate, scale, wn)]
    xr, hr, wr, gr, sr, nr = leaves
    norm = lambda v, f: v / (v.square().mean(1, keepdim=True) + 1e-4).sqrt() * f
    yr = xr + sr * gr[torch.arange(N, device="cuda") // rpg] * keep * norm(hr, wr)
    ur = norm(yr, nr)
    want = torch.autograd.grad((yr * gy.double()).sum() + (ur * gu.double()).sum(), leaves)
    assert _rel(y, yr.detach()) <= _tol(dtype, 1) and _rel(u, ur.detach()) <= _tol(dtype, 1)
    for got, wt in zip(grads, want):
        assert _rel(got, wt) <= _tol(dtype, 3)          # y is read back rounded
    into = x.clone()
    y2, u2, _ = plan.residual(into, h, w, out=into, **kw)
    assert y2.data_ptr() == into.data_ptr() and torch.equal(y, y2) and torch.equal(u, u2)
    for a, b in zip(grads, plan.residual_backward(h, y, w, stats, gy, gu, **kw)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_example(dtype):
    """The operators together as a network uses them: the loss falls and the weighted products are finite."""
    torch, _ = _setup()
    spec = importlib.util.spec_from_file_location("path_weights", os.path.join(ROOT, "examples", "path_weights.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    losses, weights, z = mod.main(pairs=300, steps=20, L=3, channels=2, dtype=dtype)
    assert losses[-1] < 0.9 * losses[0] and weights.isfinite().all() and z.isfinite().all()
    assert z.shape == (300, 2, 256)


def test_current_device_is_the_tensors(monkeypatch):
    """Kernels start on the current device: tensors of another one are refused."""
    torch, lib = _setup()
    from paper_2602_21466_amd import _ffn
    x = torch.ones(2, 8, device="cuda")
    plan = lib.NormPlan(8)
    _, rstd = plan.forward(x)
    block, w_in, w_out = lib.FfnPlan(8, 8, 8), torch.ones(16, 8, device="cuda"), torch.ones(8, 8, device="cuda")
    calls = (lambda: plan.forward(x), lambda: plan.residual(x, x), lambda: lib.dropout(x, 0.5, seed=1),
             lambda: plan.backward(x, None, rstd, x), lambda: block.forward(x, w_in, w_out))
    for call in calls:
        call()
    monkeypatch.setattr(_ffn._t, "current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
