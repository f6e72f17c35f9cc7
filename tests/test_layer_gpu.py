"""The layer norm (include/ffn.h) on the GPU against its definition in 64 bits.

Tolerances, value by value.  With h half a step of the arrays' type (eps / 2) and q = 2^-24 that of 32 bits: a result is
rounded once (h |u|; in fp16 below the normal values 2^-25).  A sum of D terms is taken by at most D / 256 + 32
additions one after another (a thread's own, then a tree), so it is off by g = (D / 256 + 32) q of the sum of magnitudes.
The variance, a sum of squares, is off by g of itself, its root and r by less; mean and n by g of the spread; with n's
own roundings 4 g (1 + |n|) covers n, and the same factor the products with it.  Sums over rows have at most
min(N, N / 256 + 64) additions in line.
"""
import pytest

pytestmark = pytest.mark.gpu

Q = 2.0 ** -24


def _setup():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_21466_amd as lib
    return torch, lib


def _dt(torch, dtype):
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]


def _inputs(torch, N, D, dtype, mean=0.5, seed=0):
    g = torch.Generator().manual_seed(100 + seed)
    t = _dt(torch, dtype)
    r = lambda *s, scale=1.0, mean=0.0: (torch.randn(*s, generator=g, dtype=torch.float64) * scale + mean).to(t)
    return r(N, D, mean=mean), r(D, scale=0.2, mean=1.0), r(D, scale=0.2), r(N, D)


def _half(torch, t):
    return torch.finfo(t).eps / 2


def _check(torch, got, want, slack, what):
    """|got - want| <= h |want| + slack, all in 64 bits."""
    t = got.dtype
    tiny = 2.0 ** -25 if t == torch.float16 else 2.0 ** -130
    got = got.double().cpu()
    worst = ((got - want).abs() - (_half(torch, t) * want.abs() + slack + tiny)).max() if want.numel() else -1.0
    assert float(worst) <= 0.0, (what, float(worst))


def _definition(torch, x, w, b, gu, eps):
    x, w, b, gu = (t.double() for t in (x, w, b, gu))
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / (c.square().mean(1, keepdim=True) + eps).sqrt()
    n, a = c * r, gu * w
    ma, man = a.mean(1, keepdim=True), (a * n).mean(1, keepdim=True)
    return {"u": n * w + b, "gx": r * (a - ma - n * man), "gw": (gu * n).sum(0), "gb": gu.sum(0), "n": n, "a": a, "r": r,
            "man": (a * n).abs().mean(1, keepdim=True), "ma": a.abs().mean(1, keepdim=True), "m": x.mean(1)}


def _compare(torch, lib, x, w, b, gu, u, stats, grads, eps, what):
    N, D = x.shape
    d = _definition(torch, x, w, b, gu, eps)
    g = (D / 256 + 32) * Q
    n1 = 1 + d["n"].abs()
    _check(torch, u, d["u"], 6 * g * (w.double().abs() * n1 + b.double().abs()), what + " u")
    spread = (x.double() - x.double().mean(1, keepdim=True)).abs().mean(1)
    _check(torch, stats[0], d["m"], g * spread + 2 * Q * d["m"].abs(), what + " mean")
    _check(torch, stats[1], d["r"][:, 0], 4 * g * d["r"][:, 0], what + " r")
    gx, gw, gb = grads
    _check(torch, gx, d["gx"], 8 * g * d["r"] * (d["a"].abs() + d["ma"] + n1 * (d["man"] + d["ma"])), what + " gx")
    rows = (min(N, N / 256 + 64) + 8) * Q
    absgu = gu.double().abs()
    _check(torch, gw, d["gw"], rows * (absgu * d["n"].abs()).sum(0) + 4 * g * (absgu * n1).sum(0), what + " gw")
    _check(torch, gb, d["gb"], rows * absgu.sum(0), what + " gb")


SIZES = [(1, 1), (5, 3), (300, 7), (33, 8), (1, 9), (40, 15), (1000, 64), (7, 65), (513, 100), (129, 289), (64, 512),
         (700, 520), (2, 1000), (31, 1089), (3, 1537), (9, 2048), (1, 4096), (5, 5000), (4, 8191), (3, 16384),
         (2, 16385), (2, 40001), (4097, 24), (1100, 200)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D", SIZES)
def test_forward_and_gradients(N, D, dtype):
    torch, lib = _setup()
    x, w, b, gu = _inputs(torch, N, D, dtype, seed=N)
    plan = lib.LayerNormPlan(D, dtype=dtype)
    dx, dw, db, dgu = (t.cuda() for t in (x, w, b, gu))
    u, stats = plan.forward(dx, dw, db)
    _compare(torch, lib, x, w, b, gu, u, stats.cpu(), plan.backward(dx, dw, stats, dgu), plan.eps, "%d x %d" % (N, D))


@pytest.mark.parametrize("N,D", [(50, 300), (20, 4096), (3, 17000)])
@pytest.mark.parametrize("mean", [1e4, -3e6])
def test_rows_far_from_zero(N, D, mean):
    """Rows whose mean is up to 2^21 times their spread: the mean's own rounding must not show."""
    torch, lib = _setup()
    x, w, b, gu = _inputs(torch, N, D, "fp32", mean=mean)
    plan = lib.LayerNormPlan(D)
    dx, dw, db, dgu = (t.cuda() for t in (x, w, b, gu))
    u, stats = plan.forward(dx, dw, db)
    _compare(torch, lib, x, w, b, gu, u, stats.cpu(), plan.backward(dx, dw, stats, dgu), plan.eps, "mean %g" % mean)


@pytest.mark.parametrize("D", [5, 96, 1089, 20000])
def test_constant_rows_and_no_parameters(D):
    torch, lib = _setup()
    plan = lib.LayerNormPlan(D, eps=1e-3)
    x = torch.full((6, D), 3.7, device="cuda")
    u, stats = plan.forward(x)
    # mean and d together give each value to a rounding: what is left is at most 2^-24 |x|, times 1 / sqrt(eps)
    assert float(u.abs().max()) <= 4 * Q * 3.7 * 1e-3 ** -0.5
    y = torch.randn(6, D, generator=torch.Generator().manual_seed(1)).cuda()
    ones, zeros = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    (u0, s0), (u1, s1) = plan.forward(y), plan.forward(y, ones, zeros)
    assert torch.equal(u0, u1) and torch.equal(s0, s1)
    for a, c in zip(plan.backward(y, None, s0, y), plan.backward(y, ones, s0, y)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D", [(9, 40), (30, 77), (5, 1089), (3, 17001), (1, 5)])
def test_strided_unaligned_in_place_and_other_stream(N, D, dtype):
    """Rows inside wider ones from an odd first column, in place, on another stream: the same bits as from packed rows."""
    torch, lib = _setup()
    x, w, b, gu = (t.cuda() for t in _inputs(torch, N, D, dtype))
    plan = lib.LayerNormPlan(D, dtype=dtype)
    u, stats = plan.forward(x, w, b)
    grads = plan.backward(x, w, stats, gu)
    wide = torch.full((N, D + 9), float("nan"), dtype=x.dtype, device="cuda")
    gwide, out = wide.clone(), wide.clone()
    wide[:, 3:3 + D], gwide[:, 1:1 + D] = x, gu
    u2, stats2 = plan.forward(wide[:, 3:3 + D], w, b, out=out[:, 5:5 + D])
    assert torch.equal(out[:, 5:5 + D], u) and torch.equal(stats, stats2)
    assert out[:, :5].isnan().all() and out[:, 5 + D:].isnan().all()
    for a, c in zip(plan.backward(wide[:, 3:3 + D], w, stats, gwide[:, 1:1 + D]), grads):
        assert torch.equal(a, c)
    again = x.clone()
    assert plan.forward(again, w, b, out=again)[0] is again and torch.equal(again, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    u3, stats3 = plan.forward(x, w, b, stream=side)
    g3 = plan.backward(x, w, stats3, gu, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(u3, u) and all(torch.equal(a, c) for a, c in zip(g3, grads))


@pytest.mark.parametrize("N,D", [(70, 48), (70, 300), (5, 20000)])
def test_single_gradients_and_determinism(N, D):
    torch, lib = _setup()
    x, w, b, gu = (t.cuda() for t in _inputs(torch, N, D, "bf16"))
    plan = lib.LayerNormPlan(D, dtype="bf16")
    _, stats = plan.forward(x, w, b)
    whole = plan.backward(x, w, stats, gu)
    for k in range(3):
        need = [j == k for j in range(3)]
        part = plan.backward(x, w, stats, gu, *need)
        assert [p is not None for p in part] == need and torch.equal(part[k], whole[k])
    assert plan.backward(x, w, stats, gu, False, False, False) == (None, None, None)


@pytest.mark.parametrize("D", [6, 64, 1089, 20000])
def test_rows_do_not_mix(D):
    torch, lib = _setup()
    x, w, b, gu = (t.cuda() for t in _inputs(torch, 40, D, "fp32"))
    plan = lib.LayerNormPlan(D)
    u, stats = plan.forward(x, w, b)
    gx = plan.backward(x, w, stats, gu, True, False, False)[0]
    bad = x.clone()
    bad[7, D // 2], bad[21] = float("inf"), float("nan")
    u2, stats2 = plan.forward(bad, w, b)
    gx2 = plan.backward(bad, w, stats2, gu, True, False, False)[0]
    keep = [i for i in range(40) if i not in (7, 21)]
    assert torch.equal(u2[keep], u[keep]) and torch.equal(gx2[keep], gx[keep])
    assert u2[7].isnan().all() and u2[21].isnan().all() and gx2[[7, 21]].isnan().all()


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_no_rows(dtype):
    torch, lib = _setup()
    plan = lib.LayerNormPlan(24, dtype=dtype)
    t = _dt(torch, dtype)
    x, w = torch.empty(0, 24, dtype=t, device="cuda"), torch.ones(24, dtype=t, device="cuda")
    u, stats = plan.forward(x, w, w)
    assert u.shape == (0, 24) and stats.shape == (2, 0)
    gx, gw, gb = plan.backward(x, w, stats, x)
    assert gx.shape == (0, 24) and not gw.any() and not gb.any()
    assert plan.backward(x, w, stats, x, True, False, False)[0].shape == (0, 24)


def test_gradients_against_differences():
    """Central differences along random directions in fp32, step 2^-6 of each argument's size: third-order terms of about
    2^-12 and rounding of 2^-24 2^6 of |u|."""
    torch, lib = _setup()
    x, w, b, gu = _inputs(torch, 11, 37, "fp32")
    plan = lib.LayerNormPlan(37)
    args = [t.cuda() for t in (x, w, b)]
    _, stats = plan.forward(*args)
    grads = plan.backward(args[0], args[1], stats, gu.cuda())
    g = torch.Generator().manual_seed(5)
    for k in range(3):
        d = torch.randn(args[k].shape, generator=g).cuda()
        d = d / d.norm() * args[k].norm()
        h = 2.0 ** -6
        up, dn = list(args), list(args)
        up[k], dn[k] = args[k] + h * d, args[k] - h * d
        num = float(((plan.forward(*up)[0].double() - plan.forward(*dn)[0].double()) * gu.cuda().double()).sum()) / (2 * h)
        ana = float((grads[k].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-3 * float(grads[k].double().norm() * d.double().norm())


def test_captured_and_replayed():
    """Forward and backward in one graph, replayed on new inputs with eager calls between."""
    torch, lib = _setup()
    plan = lib.LayerNormPlan(1089, dtype="bf16")
    sets = [[t.cuda() for t in _inputs(torch, 300, 1089, "bf16", seed=s)] for s in range(4)]
    x, w, b, gu = (t.clone() for t in sets[0])

    def step(x, w, b, gu):
        u, stats = plan.forward(x, w, b)
        return (u,) + plan.backward(x, w, stats, gu)

    step(x, w, b, gu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, w, b, gu)
    for s in sets:
        for to, fr in zip((x, w, b, gu), s):
            to.copy_(fr)
        graph.replay()
        want = step(*s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want))


def test_refusals():
    torch, lib = _setup()
    plan = lib.LayerNormPlan(32, dtype="bf16")
    x = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(32, dtype=torch.bfloat16, device="cuda")
    _, stats = plan.forward(x, w)
    for bad in (x.float(), x[:, :16], x.cpu(), x[0], x.t().contiguous().t(), torch.zeros(8, 32, dtype=x.dtype, device="cuda").as_strided((4, 32), (16, 1))):
        with pytest.raises(ValueError):
            plan.forward(bad, w)
    for bad in (w.float(), w[:16], w.cpu(), torch.ones(64, dtype=w.dtype, device="cuda")[::2]):
        with pytest.raises(ValueError):
            plan.forward(x, bad)
        with pytest.raises(ValueError):
            plan.forward(x, w, bad)
    with pytest.raises(ValueError):
        plan.backward(x, w, stats[:, :2], x)
    with pytest.raises(ValueError):
        plan.backward(x, w, stats, x[:2])
    with pytest.raises(lib.CgtpError):   # rows of the output inside the input's
        big = torch.zeros(5, 32, dtype=torch.bfloat16, device="cuda")
        plan.forward(big[:4], w, out=big[1:])
    with pytest.raises(ValueError):
        plan.backward(x, w, stats, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
