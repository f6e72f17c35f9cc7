"""The feed-forward sublayer where single values, views and the division of rows tell: bounds that hold for every value
and not in the mean of many, arrays that lie in one another's gaps or in place of one another, and plans that differ in
what a call does not read."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _setup():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_21466_amd as lib
    return torch, lib


def _dt(torch, dtype):
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]


def _randn(torch, seed, shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float64).to(_dt(torch, dtype))


# ---------------------------------------------------------------- the division of rows

@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D", [(5000, 300), (4100, 1401), (700, 20001), (3000, 4)])
def test_norm_before_does_not_depend_on_the_gate_rows(N, D, dtype):
    """A plan's rows_per_gate is about a gate: the norm before a block divides its rows in the same way, and so gives the
    same bits, whatever it is."""
    torch, lib = _setup()
    x, gu, w = _randn(torch, 1, (N, D), dtype), _randn(torch, 2, (N, D), dtype), _randn(torch, 3, (D,), dtype)
    plan = lib.NormPlan(D, dtype=dtype)
    u, rstd = plan.forward(x, w)
    want = plan.backward(x, w, rstd, gu)
    for rpg in (7, 512, N, 1 << 40):
        other = lib.NormPlan(D, dtype=dtype, rows_per_gate=rpg)
        u2, rstd2 = other.forward(x, w)
        assert torch.equal(u, u2) and torch.equal(rstd, rstd2)
        assert all(torch.equal(a, b) for a, b in zip(want, other.backward(x, w, rstd, gu))), rpg


# ---------------------------------------------------------------- 32-bit products, value by value

# Significands of which cutting or rounding at 8 and at 16 bits leaves the most, and random ones of one sign: what a
# product leaves out adds up instead of averaging out.
ONE_STEP = 2.0 ** -22 + 2.0 ** -23 * 17 / 16


@pytest.mark.parametrize("N,di,df", [(96, 8, 24), (300, 5, 130), (1030, 30, 516)])
@pytest.mark.parametrize("bits", [0x3F80FFFF, 0x3F80FF80, 0x3F80FE80, 0x3F80FE7F, 0x3F808001, 0x3FFFFFFF, None])
def test_products_of_one_sign_in_32_bits(N, di, df, bits):
    """G and U of at most 32 terms, one step of the products: 2^-22 of |x| |w| left out, one rounding of the sum with the
    last and largest of the six products, 2^-23 if it is by cutting, and a sixteenth of that for the roundings before,
    of sums of at most 2^-6 of its size."""
    torch, lib = _setup()
    if bits is None:
        g = torch.Generator(device="cuda").manual_seed(N)
        draw = lambda *s: 1.0 + torch.rand(s, generator=g, device="cuda")
    else:
        draw = lambda *s: torch.full(s, np.uint32(bits).view(np.float32).item(), device="cuda")
    x, wi, wo = draw(N, di), draw(2 * df, di), draw(8, df)
    _, saved = lib.FfnPlan(di, df, 8, activation="relu").forward(x, wi, wo, save=True)
    want = x.double() @ wi.double().T
    assert float(((saved.double() - want).abs() / want).max()) <= ONE_STEP


@pytest.mark.parametrize("bits", [0x3F80FFFF, 0x3F80FF80, 0x3F80FE80])
def test_gradient_products_of_one_sign_in_32_bits(bits):
    """grad_w_out = grad_y^T H with H = U (ReLU, G = 1), one step of 31 rows; both arrays are read by columns."""
    torch, lib = _setup()
    N, di, df, do = 31, 8, 64, 40
    v = np.uint32(bits).view(np.float32).item()
    one = lambda *s: torch.full(s, v, device="cuda")
    saved = one(N, 2 * df)
    saved[:, :df] = 1.0
    plan = lib.FfnPlan(di, df, do, activation="relu")
    gwo = plan.backward(one(N, di), one(2 * df, di), one(do, df), saved, one(N, do))[2]
    want = N * v * v
    assert float((gwo.double() - want).abs().max()) / want <= ONE_STEP


def test_products_of_the_largest_values_in_32_bits():
    """Values up to the largest of the type times small ones: finite, and as exact as others."""
    torch, lib = _setup()
    top = torch.finfo(torch.float32).max
    for s in (1.0, -1.0):
        x = torch.full((100, 8), s * top, device="cuda")
        x[1::2] *= 0.997
        x[2::3] *= 1.0 - 2.0 ** -9
        wi, wo = torch.full((16, 8), 1.1e-38, device="cuda"), torch.ones(8, 8, device="cuda")
        wi[3:9] *= 0.75
        _, saved = lib.FfnPlan(8, 8, 8, activation="relu").forward(x, wi * 2.0 ** 20, wo, save=True)
        want = x.double() @ (wi * 2.0 ** 20).double().T
        assert float(((saved.double() - want).abs() / want.abs()).max()) <= ONE_STEP


# ---------------------------------------------------------------- activations, value by value

@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N", [9, 400])
def test_activations_value_by_value(N, act, dtype):
    """H = act(G) U and dG = U act'(G) with G given and U a power of two, through weights of ones: each is the
    definition's value rounded once, to within a sixteenth of a rounding, also where the gate has nearly closed.  In 32
    bits 2^-18 for the elementary functions, and for GELU 2^-23 of G for the error function's rounding beside 1."""
    torch, lib = _setup()
    tdt = _dt(torch, dtype)
    low = -5.75 if dtype == "fp16" else -12.0            # (act(G) U stays a normal number of its type)
    g = torch.linspace(low, 4.0, N, dtype=torch.float64, device="cuda").to(tdt)
    size = 8192.0
    x = torch.stack([g, torch.ones_like(g)], 1)
    wi = torch.zeros(16, 2, dtype=tdt, device="cuda")
    wi[:8, 0], wi[8:, 1] = 1.0, size
    eye = torch.eye(8, dtype=tdt, device="cuda")
    plan = lib.FfnPlan(2, 8, 8, dtype=dtype, activation=act)
    y, saved = plan.forward(x, wi, eye, save=True)
    assert torch.equal(saved[:, 0], g.float()) and bool((saved[:, 8:] == size).all())
    gy = torch.zeros(N, 8, dtype=tdt, device="cuda")
    gy[:, 0] = 1.0
    gx = plan.backward(x, wi, eye, saved, gy, True, False, False)[0]
    v = g.double()
    if act == "silu":
        s = torch.sigmoid(v)
        a, da = v * s, s * (1.0 + v * (1.0 - s))
    else:
        cdf = 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)     # (ndtr cancels beside 1 here)
        a, da = v * cdf, cdf + v * torch.exp(-0.5 * v * v) / (2.0 * np.pi) ** 0.5
    tol = {"fp32": 2.0 ** -18, "bf16": 2.0 ** -8 * 17 / 16, "fp16": 2.0 ** -11 * 17 / 16}[dtype]
    slack = 2.0 ** -23 if dtype == "fp32" and act == "gelu" else 0.0
    assert bool(((y.double() / size - a[:, None]).abs() <= tol * a[:, None].abs() + slack * v[:, None].abs()).all())
    # (the derivative passes zero about G = -0.75 or -1.28, where its two terms, of 0.2 or more, cancel)
    crossing = (v > -1.6) & (v < -0.5)
    part = torch.where(crossing, da.abs().clamp_min(0.01), da.abs())
    assert bool(((gx[:, 0].double() / size - da).abs() <= tol * part + slack).all())


# ---------------------------------------------------------------- few rows

@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", [3, 24, 40])
@pytest.mark.parametrize("di,df,do", [(40, 70, 3100), (70, 3100, 40), (40, 16420, 24)])
def test_few_rows_by_every_number_of_weight_rows(N, di, df, do, dtype):
    """8, 16 and 32 weight rows a work-group, in both products: against 64 bits, H and the output rounded once each."""
    torch, lib = _setup()
    x, wi, wo = _randn(torch, N, (N, di), dtype), _randn(torch, 2, (2 * df, di), dtype), _randn(torch, 3, (do, df), dtype)
    wi, wo = wi * di ** -0.5, wo * df ** -0.5
    y, saved = lib.FfnPlan(di, df, do, dtype=dtype).forward(x, wi, wo, save=True)
    z = x.double() @ wi.double().T
    want = (torch.nn.functional.silu(z[:, :df]) * z[:, df:]) @ wo.double().T
    unit = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    assert float((saved.double() - z).norm() / z.norm()) <= 4e-6
    assert float((y.double() - want).norm() / want.norm()) <= 2 * unit + 4e-6


# ---------------------------------------------------------------- views and arrays in place of others

def test_one_row_of_a_wide_array():
    """The stride of a single row is never used: a row of an array of any width is taken."""
    torch, lib = _setup()
    big = torch.zeros(3, (1 << 21) + 64, dtype=torch.bfloat16, device="cuda")
    x = big[1:2, 5:69]
    x.copy_(_randn(torch, 1, (1, 64), "bf16"))
    packed = x.clone()
    wi, wo = _randn(torch, 2, (96, 64), "bf16"), _randn(torch, 3, (64, 48), "bf16")
    plan, norm = lib.FfnPlan(64, 48, 64, dtype="bf16"), lib.NormPlan(64, dtype="bf16")
    y, saved = plan.forward(x, wi, wo, save=True)
    assert torch.equal(y, plan.forward(packed, wi, wo))
    for a, b in zip(plan.backward(x, wi, wo, saved, x), plan.backward(packed, wi, wo, saved, packed)):
        assert torch.equal(a, b)
    u, rstd = norm.forward(x)
    assert torch.equal(u, norm.forward(packed)[0])
    assert torch.equal(norm.backward(x, None, rstd, x)[0], norm.backward(packed, None, rstd, packed)[0])
    assert torch.equal(lib.dropout(x, 0.5, seed=1), lib.dropout(packed, 0.5, seed=1))


def test_columns_of_one_array_side_by_side():
    """An input and an output that are neighbouring columns of one array do not overlap; columns that meet do."""
    torch, lib = _setup()
    N, D = 37, 45
    for width, at in ((2 * D, D), (2 * D + 9, D + 4), (3 * D, 2 * D)):
        buf = torch.full((N, width), 7.0, device="cuda")
        x, out = buf[:, :D], buf[:, at:at + D]
        x.copy_(_randn(torch, width, (N, D), "fp32"))
        packed = x.clone()
        rest = torch.ones(width, dtype=torch.bool)
        rest[:D] = rest[at:at + D] = False
        norm = lib.NormPlan(D)
        for call in (lambda a, **k: norm.forward(a, **k)[0], lambda a, **k: lib.dropout(a, 0.25, seed=5, **k)):
            for a, b in ((x, out), (out, x)):
                a.copy_(packed)
                assert torch.equal(call(a, out=b), call(packed)) and torch.equal(a, packed)
                assert bool((buf[:, rest] == 7.0).all())
        for bad in (buf[:, at - 1:at - 1 + D] if at == D else buf[:, D - 1:2 * D - 1], buf[:, 1:D + 1]):
            with pytest.raises(lib.CgtpError):
                norm.forward(x, out=bad)
            with pytest.raises(lib.CgtpError):
                lib.dropout(x, 0.25, seed=5, out=bad)
    # the output's rows begin inside the input's, and end in the row after
    buf = torch.zeros(N + 1, 2 * D, device="cuda").reshape(-1)
    x = torch.as_strided(buf, (N, D), (2 * D, 1), 0)
    late = torch.as_strided(buf, (N, D), (2 * D, 1), D + 1)
    with pytest.raises(lib.CgtpError):
        lib.NormPlan(D).forward(x, out=late)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D", [(300, 40), (700, 1029), (400, 1401), (130, 5001), (90, 9001), (20, 5)])
def test_results_in_place_of_inputs(N, D, dtype):
    """u in place of x, and (by the C entry) grad_x in place of grad_y, also where two threads share columns: the same
    bits as elsewhere."""
    torch, lib = _setup()
    x, h, gy, gu, gate = (_randn(torch, k, (N, D), dtype) for k in range(5))
    w, scale, wn = (_randn(torch, 9 + k, (D,), dtype) for k in range(3))
    plan = lib.NormPlan(D, dtype=dtype, dropout=0.25)
    want, rstd = plan.forward(x, w)
    into = x.clone()
    got, rstd2 = plan.forward(into, w, out=into)
    assert got is into and torch.equal(want, into) and torch.equal(rstd, rstd2)
    kw = {"gate": gate, "scale": scale, "w_next": wn, "seed": 3, "offset": 8}
    y, u, stats = plan.residual(x, h, w, **kw)
    norm = lib.ffn_norm(D, 1, {"fp32": lib.FFN_FP32, "bf16": lib.FFN_BF16, "fp16": lib.FFN_FP16}[dtype], 1e-6, 0.25, 3, 8)
    need = lib.ffn_norm_workspace_bytes(norm, N, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    p = lambda t: None if t is None else t.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    for last in (gu, None):
        want = plan.residual_backward(h, y, w, stats, gy, last, **kw)
        gx = gy.clone()
        rest = [torch.empty_like(t) for t in (h, w, gate, scale, wn)]
        lib.ffn_residual_backward(norm, p(h), p(y), p(w), p(gate), p(scale), p(wn), p(stats), p(gx), p(last), p(gx),
                                  p(rest[0]), p(rest[1]), p(rest[2]), p(rest[3]), p(rest[4]), N, p(ws), need, stream)
        for a, b in zip(want, [gx] + rest):
            assert torch.equal(a, b)
