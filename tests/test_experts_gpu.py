"""The experts' gated blocks (include/experts.h) on the GPU against their definition in 64 bits, and a run of the
operators around them together.

Tolerances, value by value, by following each rounding through the products.  With h half a step of the arrays' type and
q = 2^-24: a sum of K products is off by at most s(K) = (K / 16 + 40) q of the sum of magnitudes (the matrix
instructions add 16 or 32 of them at once), in fp32 and 2^-22 more, which is what its bf16 parts leave out.  G and U are
such sums.  The activations are off by 2^-20, gelu's error function by 4e-5 of its own value, in 16-bit arrays, and by 8 q
in fp32; their slopes are below 1.2 and the slopes of those below 1.  H, dG and dU are rounded to the arrays' type between
the products, and every result once.  Where relu's slope jumps within G's error, dG may be either value.
"""
import math

import numpy as np
import pytest

from test_routes_gpu import _index, _order

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


def _act64(torch, name, g):
    """act(g), act'(g)."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    return g.clamp_min(0), (g > 0).double()


def _case(torch, N, K, E, di, df, do, dtype, kind, seed=0):
    g = torch.Generator().manual_seed(seed + N)
    t = _dt(torch, dtype)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g, dtype=torch.float64) * scale).to(t)
    return _index(N, K, E, kind, seed), r(N, di), r(E, 2 * df, di, scale=di ** -0.5), r(E, do, df, scale=df ** -0.5), r(N * K, do)


def _reference(torch, index, x, w_in, w_out, gy, act):
    """{name: (value, bound)} in 64 bits; rows of no expert are left out of y, z (saved) and the bounds."""
    N, K = index.shape
    E, df = w_in.shape[0], w_out.shape[2]
    di, do = x.shape[1], w_out.shape[1]
    place, source, offsets = _order(index, E)
    t = x.dtype
    h, wide = torch.finfo(t).eps / 2, t == torch.float32
    tiny = 2.0 ** -25 if t == torch.float16 else 0.0
    s = lambda k: (k / 16 + 40) * Q + (2.0 ** -22 if wide else 0.0)
    ea = 8 * Q if wide else 5e-5
    x, w_in, w_out, gy = (v.double() for v in (x, w_in, w_out, gy))
    M = int(offsets[-1])
    out = {k: (torch.zeros(*n, dtype=torch.float64), torch.zeros(*n, dtype=torch.float64)) for k, n in
           (("y", (M, do)), ("z", (M, 2 * df)), ("gx", (N, di)), ("gw_in", w_in.shape), ("gw_out", w_out.shape))}

    def put(name, at, value, slack):
        out[name][0][at] = value
        out[name][1][at] = slack

    for e in range(E):
        a, b = int(offsets[e]), int(offsets[e + 1])
        token = torch.from_numpy(source[a:b] // K)
        X, W, Wo, G_y = x[token], w_in[e], w_out[e], gy[a:b]
        aX, aW, aWo, aGy = X.abs(), W.abs(), Wo.abs(), G_y.abs()
        z = X @ W.T
        dz = s(di) * (aX @ aW.T)
        put("z", slice(a, b), z, dz)
        g, u, eg, eu = z[:, :df], z[:, df:], dz[:, :df], dz[:, df:]
        v, dv = _act64(torch, act, g)
        H = v * u
        eH = 1.2 * eg * (u.abs() + eu) + v.abs() * eu + ea * (g.abs() * u.abs())
        eH = eH + h * (H.abs() + eH) + tiny
        y = H @ Wo.T
        ey = eH @ aWo.T + s(df) * ((H.abs() + eH) @ aWo.T)
        put("y", slice(a, b), y, ey + h * (y.abs() + ey) + tiny)
        dH = G_y @ Wo
        edH = s(do) * (aGy @ aWo)
        edv = eg + ea + 4 * Q * g.abs()
        if act == "relu":
            edv = (g.abs() <= eg).double()
        dU, dG = dH * v, dH * u * dv
        edU = edH * v.abs() + (dH.abs() + edH) * (1.2 * eg + ea * g.abs())
        edG = edH * (u * dv).abs() + (dH.abs() + edH) * ((u.abs() + eu) * edv + eu * dv.abs())
        D, eD = torch.cat([dG, dU], 1), torch.cat([edG, edU], 1)
        eD = eD + 4 * Q * D.abs()
        eD = eD + h * (D.abs() + eD) + tiny
        aD = D.abs() + eD
        gxs, egxs = D @ W, eD @ aW + s(2 * df) * (aD @ aW)
        out["gx"][0].index_add_(0, token, gxs)
        out["gx"][1].index_add_(0, token, egxs + (K + 1) * Q * gxs.abs())
        gw = D.T @ X
        put("gw_in", e, gw, eD.T @ aX + s(b - a) * (aD.T @ aX))
        gw = G_y.T @ H
        put("gw_out", e, gw, aGy.T @ eH + s(b - a) * (aGy.T @ (H.abs() + eH)))
    for k in ("gx", "gw_in", "gw_out"):
        v, e = out[k]
        out[k] = (v, e + h * (v.abs() + e) + tiny)
    out["z"] = (out["z"][0], out["z"][1] + Q * out["z"][0].abs())
    return out, M


def _check(got, pair, what):
    want, slack = pair
    got = got.double().cpu()
    assert got.shape == want.shape and bool(got.isfinite().all()), what
    over = ((got - want).abs() - slack - 2.0 ** -130)
    assert not over.numel() or float(over.max()) <= 0.0, (what, float(over.max()))


# rows, choices, experts and sizes: one row, few rows, runs that end inside tiles, odd strides, long sums, wide outputs, one
# product by the kernels for few rows and the other by tiles, both ways
SIZES = [(1, 1, 1, 1, 1, 1), (1, 2, 8, 64, 128, 64), (1, 1, 3, 81, 324, 489), (3, 2, 4, 17, 5, 31), (16, 4, 6, 256, 64, 256),
         (17, 1, 2, 96, 200, 40), (64, 2, 3, 128, 64, 8), (100, 3, 5, 75, 130, 77), (200, 2, 65, 40, 72, 24),
         (300, 2, 3, 264, 72, 129), (257, 1, 1, 520, 264, 136), (500, 4, 4, 64, 256, 320), (1000, 1, 7, 32, 48, 56),
         (90, 2, 200, 24, 16, 9), (33, 2, 2, 1000, 2056, 8), (600, 1, 2, 8, 8, 2000), (40, 1, 1, 64, 61, 24),
         (80, 1, 2, 61, 64, 24), (16, 1, 4, 2000, 2056, 1032)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,K,E,di,df,do", SIZES)
@pytest.mark.parametrize("kind", ["even", "some", "skewed"])
def test_forward_and_gradients(N, K, E, di, df, do, dtype, kind):
    torch, lib = _setup()
    act = ("silu", "gelu", "relu")[(N + di) % 3]
    index, x, wi, wo, gy = _case(torch, N, K, E, di, df, do, dtype, kind)
    ref, M = _reference(torch, index, x, wi, wo, gy, act)
    gy[M:] = float("nan")   # rows behind the last are not read
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype, activation=act)
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    dx, dwi, dwo, dgy = (t.cuda() for t in (x, wi, wo, gy))
    out = torch.full((N * K, do), 7.0, dtype=x.dtype, device="cuda")
    y = plan.forward(dx, routes, dwi, dwo, out=out)
    assert y is out and (y[M:] == 7.0).all()   # nor written
    y2, saved = plan.forward(dx, routes, dwi, dwo, save=True)
    assert torch.equal(y[:M], y2[:M])
    _check(y[:M], ref["y"], "y")
    _check(saved[:M], ref["z"], "saved")
    for got, name in zip(plan.backward(dx, routes, dwi, dwo, saved, dgy), ("gx", "gw_in", "gw_out")):
        assert got.dtype == x.dtype
        _check(got, ref[name], name)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["one", "none"])
@pytest.mark.parametrize("N", [2, 300])
def test_one_expert_takes_all_or_none(N, kind, dtype):
    torch, lib = _setup()
    index, x, wi, wo, gy = _case(torch, N, 2, 70, 48, 40, 24, dtype, kind)
    ref, M = _reference(torch, index, x, wi, wo, gy, "silu")
    wi[:-1], wo[:-1] = float("nan"), float("nan")   # weights of experts without rows are not read
    plan = lib.ExpertsPlan(70, 48, 40, 24, dtype=dtype)
    routes = lib.Routes(torch.from_numpy(index).cuda(), 70)
    dx, dwi, dwo, dgy = (t.cuda() for t in (x, wi, wo, gy))
    y, saved = plan.forward(dx, routes, dwi, dwo, save=True)
    _check(y[:M], ref["y"], "y")
    for got, name in zip(plan.backward(dx, routes, dwi, dwo, saved, dgy), ("gx", "gw_in", "gw_out")):
        _check(got, ref[name], name)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", [1, 20, 150])
@pytest.mark.parametrize("di,df,do", [(80, 64, 72), (77, 61, 35), (78, 66, 70)])
def test_strided_rows_single_gradients_and_other_stream(N, di, df, do, dtype):
    torch, lib = _setup()
    K, E = 2, 5
    index, x, wi, wo, gy = _case(torch, N, K, E, di, df, do, dtype, "even")
    x, wi, wo, gy = (t.cuda() for t in (x, wi, wo, gy))
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    grads = plan.backward(x, routes, wi, wo, saved, gy)
    wide = torch.full((N, di + 11), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 3:3 + di] = x
    # grad_out from an odd element on
    odd = torch.empty(gy.numel() + 1, dtype=gy.dtype, device="cuda")[1:].view_as(gy)
    odd.copy_(gy)
    y2, saved2 = plan.forward(wide[:, 3:3 + di], routes, wi, wo, save=True)
    assert torch.equal(y, y2) and torch.equal(saved, saved2)
    for a, b in zip(plan.backward(wide[:, 3:3 + di], routes, wi, wo, saved, odd), grads):
        assert torch.equal(a, b)
    for k in range(3):
        need = [j == k for j in range(3)]
        part = plan.backward(x, routes, wi, wo, saved, gy, *need)
        assert [p is not None for p in part] == need and torch.equal(part[k], grads[k])
    assert plan.backward(x, routes, wi, wo, saved, gy, False, False, False) == (None, None, None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y3, saved3 = plan.forward(x, routes, wi, wo, save=True, stream=side)
    g3 = plan.backward(x, routes, wi, wo, saved3, gy, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y3, y) and all(torch.equal(a, b) for a, b in zip(g3, grads))


@pytest.mark.parametrize("N", [12, 200])
def test_rows_and_experts_do_not_mix(N):
    """A NaN row reaches the rows of its own choices alone; NaN weights those of their expert."""
    torch, lib = _setup()
    for dtype in ("fp32", "bf16"):
        index, x, wi, wo, gy = (t.cuda() if torch.is_tensor(t) else t for t in _case(torch, N, 2, 4, 64, 96, 64, dtype, "even"))
        routes = lib.Routes(torch.from_numpy(index).cuda(), 4)
        plan = lib.ExpertsPlan(4, 64, 96, 64, dtype=dtype)
        want, saved = plan.forward(x, routes, wi, wo, save=True)
        bad = x.clone()
        bad[7] = float("nan")
        got = plan.forward(bad, routes, wi, wo)
        hit = torch.zeros(2 * N, dtype=torch.bool, device="cuda")
        hit[routes.place[7].long()] = True
        assert got[hit].isnan().all() and torch.equal(got[~hit], want[~hit])
        wbad = wi.clone()
        wbad[2] = float("nan")
        got, saved_bad = plan.forward(x, routes, wbad, wo, save=True)
        a, b = routes.offsets[2:4].tolist()
        assert got[a:b].isnan().all() and torch.equal(got[:a], want[:a]) and torch.equal(got[b:], want[b:])
        g1, g2 = plan.backward(x, routes, wi, wo, saved, gy), plan.backward(x, routes, wbad, wo, saved_bad, gy)
        for e in range(4):
            for p, q in zip(g1[1:], g2[1:]):
                assert q[e].isnan().any() if e == 2 else torch.equal(p[e], q[e])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", [9, 150, 700])
@pytest.mark.parametrize("di,df,do", [(77, 61, 35), (66, 130, 6), (131, 257, 129)])
def test_rows_that_end_inside_a_chunk_do_not_mix(N, di, df, do, dtype):
    """What lies behind a row in memory, the next row, the next expert's or the array's end, adds nothing to it, though it
    is infinite or NaN."""
    torch, lib = _setup()
    K, E = 2, 3
    index, x, wi, wo, gy = (t.cuda() if torch.is_tensor(t) else t for t in _case(torch, N, K, E, di, df, do, dtype, "even"))
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    grads = plan.backward(x, routes, wi, wo, saved, gy)
    a, b = routes.offsets[1:3].tolist()
    for bad in (float("nan"), float("inf")):
        # a row of the second expert's weights: its column of G (or U) alone, of the expert's rows alone
        for row in (1, df, 2 * df - 1):
            w = wi.clone()
            w[1, row] = bad
            got = plan.forward(x, routes, w, wo, save=True)[1]
            hit = torch.zeros(saved.shape, dtype=torch.bool, device="cuda")
            hit[a:b, row] = True
            assert not got[hit].isfinite().any() and torch.equal(got[~hit], saved[~hit])
        for row in (0, do - 1):
            w = wo.clone()
            w[1, row] = bad
            got = plan.forward(x, routes, wi, w)
            hit = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
            hit[a:b, row] = True
            assert not got[hit].isfinite().any() and torch.equal(got[~hit], y[~hit])
        # a row of grad_y: its own row's gradients
        g = gy.clone()
        g[a] = bad
        token = int(routes.source[a]) // K
        gx = plan.backward(x, routes, wi, wo, saved, g, True, False, False)[0]
        keep = [n for n in range(N) if n != token]
        assert not gx[token].isfinite().any() and torch.equal(gx[keep], grads[0][keep])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_weights_that_end_with_a_page(dtype):
    """Odd rows, in arrays whose last byte is the last of a page of memory, and in others: the same bits."""
    torch, lib = _setup()
    E, di, df, do, N = 2, 3, 512, 512, 40
    index, x, wi, wo, gy = _case(torch, N, 1, E, di, df, do, dtype, "even")
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    outs = []
    for shift in (0, 256):
        def at_page(t):
            raw = torch.zeros(t.numel() * t.element_size() + 16384, dtype=torch.uint8, device="cuda")
            end = (raw.data_ptr() + t.numel() * t.element_size() + 4095) // 4096 * 4096 + 4096 - shift
            first = end - t.numel() * t.element_size() - raw.data_ptr()
            out = raw[first:first + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
            out.copy_(t)
            return out
        a = [at_page(t.cuda()) for t in (x, wi, wo, gy)]
        assert all((t.data_ptr() + t.numel() * t.element_size()) % 4096 == (-shift) % 4096 for t in a)
        y, saved = plan.forward(a[0], routes, a[1], a[2], save=True)
        outs.append((y, saved) + plan.backward(a[0], routes, a[1], a[2], saved, a[3]))
    assert all(torch.equal(p, q) for p, q in zip(*outs))


def test_one_expert_is_the_single_block():
    """With one expert and one choice a row, rows are those of a FfnPlan up to the order of the sums."""
    torch, lib = _setup()
    _, x, wi, wo, gy = _case(torch, 300, 1, 1, 72, 136, 40, "fp32", "even")
    x, wi, wo, gy = (t.cuda() for t in (x, wi, wo, gy))
    routes = lib.Routes(torch.zeros(300, dtype=torch.int64, device="cuda"), 1)
    plan, block = lib.ExpertsPlan(1, 72, 136, 40), lib.FfnPlan(72, 136, 40)
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    y1, saved1 = block.forward(x, wi[0], wo[0], save=True)
    for a, b in zip((y, saved) + plan.backward(x, routes, wi, wo, saved, gy),
                    (y1, saved1) + block.backward(x, wi[0], wo[0], saved1, gy)):
        assert float((a.reshape(b.shape) - b).norm()) <= 4e-6 * float(b.norm())


def test_no_rows():
    torch, lib = _setup()
    plan = lib.ExpertsPlan(3, 16, 24, 8, dtype="bf16")
    t = torch.bfloat16
    routes = lib.Routes(torch.empty(0, 2, dtype=torch.int64, device="cuda"), 3)
    x, wi, wo = torch.empty(0, 16, dtype=t, device="cuda"), torch.ones(3, 48, 16, dtype=t, device="cuda"), torch.ones(3, 8, 24, dtype=t, device="cuda")
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    assert y.shape == (0, 8) and saved.shape == (0, 48)
    gx, gwi, gwo = plan.backward(x, routes, wi, wo, saved, y)
    assert gx.shape == (0, 16) and not gwi.any() and not gwo.any()
    assert plan.backward(x, routes, wi, wo, saved, y, True, False, False)[0].shape == (0, 16)


def _mixture(lib, norm, plan, x, lw, lb, index, weights, wi, wo, gy):
    """A residual mixture, forward and backward: t = x + combine(block(L(x; w, b))), through every operator."""
    u, stats = norm.forward(x, lw, lb)
    routes = lib.Routes(index, plan.experts)
    ys, saved = plan.forward(u, routes, wi, wo, save=True)
    t = x + routes.combine(ys, weights)
    gys, gweights = routes.combine_backward(ys, weights, gy)
    gu, gwi, gwo = plan.backward(u, routes, wi, wo, saved, gys)
    gx, glw, glb = norm.backward(x, lw, stats, gu)
    return t, gx + gy, glw, glb, gweights, gwi, gwo


def test_a_mixture_and_its_gradients():
    """The whole mixture in fp32 against torch in 64 bits, and against differences along random directions."""
    torch, lib = _setup()
    N, K, E, D, F = 120, 2, 6, 56, 88
    index, x, wi, wo, _ = _case(torch, N, K, E, D, F, D, "fp32", "some")
    g = torch.Generator().manual_seed(3)
    lw, lb, w, gy = (torch.randn(s, generator=g) for s in ((D,), (D,), (N, K), (N, D)))
    norm, plan = lib.LayerNormPlan(D), lib.ExpertsPlan(E, D, F, D)
    di = torch.from_numpy(index).cuda()
    dev = [t.cuda() for t in (x, lw, lb, w, wi, wo)]
    run = lambda x, lw, lb, w, wi, wo: _mixture(lib, norm, plan, x, lw, lb, di, w, wi, wo, gy.cuda())
    got = run(*dev)
    leaves = [t.double().requires_grad_(True) for t in (x, lw, lb, w, wi, wo)]
    u = torch.nn.functional.layer_norm(leaves[0], (D,), leaves[1], leaves[2], norm.eps)
    t = leaves[0]
    for k in range(K):
        rows = [n for n in range(N) if 0 <= index[n, k] < E]
        e = torch.from_numpy(index[rows, k].astype(np.int64))
        z = torch.bmm(leaves[4][e], u[rows][:, :, None])[:, :, 0]
        h = torch.nn.functional.silu(z[:, :F]) * z[:, F:]
        t = t.index_add(0, torch.tensor(rows), leaves[3][rows, k][:, None] * torch.bmm(leaves[5][e], h[:, :, None])[:, :, 0])
    want = [t.detach()] + list(torch.autograd.grad(t, leaves, gy.double()))
    # every one passes at most twelve sums in 32 bits whose parts leave out 2^-22: 12 * 2^-22 of the factors' norms
    for a, b in zip(got, want):
        assert float((a.double().cpu() - b).norm()) <= 12 * 2.0 ** -20 * float(b.norm())
    for k in range(6):
        d = torch.randn(dev[k].shape, generator=g).cuda()
        d, h = d / d.norm() * dev[k].norm(), 2.0 ** -7
        up, dn = list(dev), list(dev)
        up[k], dn[k] = dev[k] + h * d, dev[k] - h * d
        num = float(((run(*up)[0].double() - run(*dn)[0].double()) * gy.cuda().double()).sum()) / (2 * h)
        ana = float((got[k + 1].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-3 * float(got[k + 1].double().norm() * d.double().norm())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N", [3, 400])
def test_mixture_captured_and_replayed(N, dtype):
    """The mixture in two graphs that share their pool, replayed in turn on new choices and values with eager calls between."""
    torch, lib = _setup()
    K, E, D, F = 2, 5, 64, 96
    norm, plan = lib.LayerNormPlan(D, dtype=dtype), lib.ExpertsPlan(E, D, F, D, dtype=dtype)
    t = _dt(torch, dtype)

    def inputs(s):
        index, x, wi, wo, _ = _case(torch, N, K, E, D, F, D, dtype, ("even", "some", "one", "none")[s % 4], s)
        g = torch.Generator().manual_seed(s)
        lw, lb, gy = (torch.randn(n, generator=g).to(t) for n in ((D,), (D,), (N, D)))
        return [v.cuda() for v in (x, lw, lb, torch.from_numpy(index), torch.rand(N, K, generator=g), wi, wo, gy)]

    step = lambda a: _mixture(lib, norm, plan, *a)
    args = [inputs(0), inputs(1)]
    step(args[0])
    torch.cuda.synchronize()
    graphs, outs, pool = [], [], None
    for a in args:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append(step(a))
        graphs.append(graph)
        pool = graph.pool()
    for s in range(6):
        new, k = inputs(s + 2), s % 2
        for to, fr in zip(args[k], new):
            to.copy_(fr)
        graphs[k].replay()
        got = [v.clone() for v in outs[k]]
        want = step(new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), s


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N", [6, 500])
def test_entries_out_of_range_stay_inside(N, dtype):
    """An order with entries far out of their range: other results, but nothing is written outside the outputs, and rows
    that no such entry is about keep theirs."""
    torch, lib = _setup()
    K, E, di, df, do = 2, 3, 40, 56, 24
    index, x, wi, wo, gy = (t.cuda() if torch.is_tensor(t) else t for t in _case(torch, N, K, E, di, df, do, dtype, "even"))
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    good = lib.Routes(torch.from_numpy(index).cuda(), E)
    want, saved = plan.forward(x, good, wi, wo, save=True)
    want_y = good.combine(want)
    S, far = N * K, torch.tensor([-2 ** 31, 2 ** 31 - 1, N * K, -7], dtype=torch.int32, device="cuda")
    bad = lib.Routes(torch.from_numpy(index).cuda(), E)
    bad.place[1], bad.source[3:5] = far[:2], far[1:3]
    room = torch.full((S + 64, do), 7.0, dtype=x.dtype, device="cuda")
    out = plan.forward(x, bad, wi, wo, out=room[32:32 + S])
    keep = [p for p in range(S) if p not in (3, 4)]
    assert torch.equal(out[keep], want[keep]) and (room[:32] == 7).all() and (room[32 + S:] == 7).all()
    rows = [n for n in range(N) if n != 1]
    assert torch.equal(bad.combine(want)[rows], want_y[rows]) and not bad.combine(want)[1].any()
    bad.offsets[0], bad.offsets[E] = far[0], far[1]
    xs = torch.full((S + 64, di), 7.0, dtype=x.dtype, device="cuda")
    bad.gather(x, out=xs[32:32 + S])
    out = plan.forward(x, bad, wi, wo, out=room[32:32 + S])
    assert (room[:32] == 7).all() and (room[32 + S:] == 7).all() and (xs[:32] == 7).all() and (xs[32 + S:] == 7).all()
    grads = plan.backward(x, bad, wi, wo, saved, gy)
    gys, gw = bad.combine_backward(want, torch.ones(N, K, device="cuda"), want_y)
    assert all(bool(t.isfinite().all()) for t in (*grads, gw)) and not gw[1].any()


def test_refusals():
    torch, lib = _setup()
    plan = lib.ExpertsPlan(3, 16, 24, 8)
    routes = lib.Routes(torch.zeros(4, 2, dtype=torch.int64, device="cuda"), 3)
    x, wi, wo = torch.zeros(4, 16, device="cuda"), torch.zeros(3, 48, 16, device="cuda"), torch.zeros(3, 8, 24, device="cuda")
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    for bad in (x[:3], x.half(), x.cpu(), x[:, :8]):
        with pytest.raises(ValueError):
            plan.forward(bad, routes, wi, wo)
    for bad in (None, torch.zeros(4, 2, device="cuda"), lib.Routes(torch.zeros(4, 2, dtype=torch.int64, device="cuda"), 4),
                lib.Routes(torch.zeros(5, 2, dtype=torch.int64, device="cuda"), 3)):
        with pytest.raises(ValueError):
            plan.forward(x, bad, wi, wo)
    for bad in (wi[:2], wi.half(), wi.transpose(1, 2), wi.cpu()):
        with pytest.raises(ValueError):
            plan.forward(x, routes, bad, wo)
    with pytest.raises(ValueError):
        plan.forward(x, routes, wi, wo[:, :, :8])
    with pytest.raises(ValueError):
        plan.backward(x, routes, wi, wo, saved[:7], y)
    with pytest.raises(ValueError):
        plan.backward(x, routes, wi, wo, saved, y[:7])
    with pytest.raises(ValueError):
        plan.forward(x, routes, wi, wo, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(lib.CgtpError):
        plan.forward(x, routes, wi, wo, out=wi.reshape(-1)[:64].view(8, 8))
