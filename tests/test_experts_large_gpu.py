"""The experts' operators and the layer norm with offsets past 32 bits and grids of more rows than a launch takes, and
calls of one plan on two streams at once.  Tolerances as in test_experts_gpu.py, test_routes_gpu.py and test_layer_gpu.py;
of results that are too many, rows or columns are drawn and the definition is taken of those alone.
"""
import numpy as np
import pytest

from test_experts_gpu import _check, _dt, _reference, _setup
from test_layer_gpu import Q, _compare

pytestmark = pytest.mark.gpu


def _randn(torch, t, *shape, scale=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(*shape, dtype=t, device="cuda").normal_(0.0, scale, generator=g)


# x past 2^31 bytes, x's sorted rows past 2^31 values; H, dG, dU past 2^32 bytes, saved past 2^32 values; and each product in
# more than a round of 256-wide tiles, of which those beyond it are cut
@pytest.mark.parametrize("N,K,E,di,df,do,dtype", [(66001, 2, 3, 16384, 8, 8, "bf16"), (40003, 1, 2, 16385, 4, 12, "fp32"),
                                                  (100003, 2, 3, 64, 16400, 40, "bf16"), (3200, 1, 2, 520, 7399, 7402, "bf16"),
                                                  (3200, 1, 2, 519, 7402, 7399, "fp16")])
def test_long_and_wide(N, K, E, di, df, do, dtype):
    torch, lib = _setup()
    t = _dt(torch, dtype)
    rng = np.random.default_rng(N)
    index = rng.integers(-1, E, (N, K))
    x, wi, wo = _randn(torch, t, N, di, seed=1), _randn(torch, t, E, 2 * df, di, scale=di ** -0.5, seed=2), _randn(torch, t, E, do, df, scale=df ** -0.5, seed=3)
    gy = _randn(torch, t, N * K, do, seed=4)
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    y, saved = plan.forward(x, routes, wi, wo, save=True)
    assert torch.equal(plan.forward(x, routes, wi, wo)[: int(routes.offsets[-1])], y[: int(routes.offsets[-1])])
    gx, gwi, gwo = plan.backward(x, routes, wi, wo, saved, gy)
    # of some rows, the first and the last among them: y, saved and gx
    rows = np.unique(np.concatenate([rng.integers(0, N, 20), [0, N - 1], np.nonzero((index >= 0).any(1))[0][-3:]]))
    place = routes.place.cpu().numpy()[rows]
    sub = index[rows]
    order = np.argsort(np.where(sub.reshape(-1) < 0, E, sub.reshape(-1)), kind="stable")   # the sorted rows of these alone
    at = torch.from_numpy(np.where(place.reshape(-1)[order] < 0, 0, place.reshape(-1)[order])).cuda()
    ref, M = _reference(torch, sub, x[torch.from_numpy(rows).cuda()].cpu(), wi.cpu(), wo.cpu(), gy[at].cpu(), "silu")
    at = at[:M]
    _check(y[at], ref["y"], "y")
    _check(saved[at], ref["z"], "saved")
    _check(gx[torch.from_numpy(rows).cuda()], ref["gx"], "gx")
    # of some hidden columns, the first and the last among them: their weights' gradients, which are sums over all rows
    cols = torch.from_numpy(np.unique(np.concatenate([rng.integers(0, df, 3), [0, df - 1]])))
    both = torch.cat([cols, cols + df])
    z = _columns(torch, x, index, routes, wi[:, both.cuda()], wo[:, :, cols.cuda()], gy, E)
    for e in range(E):
        D, eD, X, H, eH, G = z[e]
        n = len(X)
        s = (n / 16 + 40) * Q + (2.0 ** -22 if dtype == "fp32" else 0.0)
        h = torch.finfo(t).eps / 2
        want, X = D.T @ X, X.abs()
        slack = eD.T @ X + s * ((D.abs() + eD).T @ X)
        _check(gwi[e, both.cuda()][:, -16:], (want.cpu(), (slack + h * (want.abs() + slack)).cpu()), "gw_in")
        want = G.T @ H
        slack = G.abs().T @ eH + s * (G.abs().T @ (H.abs() + eH))
        _check(gwo[e][:, cols.cuda()], (want.cpu(), (slack + h * (want.abs() + slack)).cpu()), "gw_out")


def _columns(torch, x, index, routes, wi, wo, gy, E):
    """(dG dU, bound, X's last 16 columns, H, bound, gy) of each expert's rows for some hidden columns, in 64 bits on the
    GPU; the bounds are _reference()'s."""
    t = x.dtype
    h, wide = torch.finfo(t).eps / 2, t == torch.float32
    s = lambda k: (k / 16 + 40) * Q + (2.0 ** -22 if wide else 0.0)
    ea = 8 * Q if wide else 5e-5
    K, di, do, c = index.shape[1], x.shape[1], gy.shape[1], wo.shape[2]
    out, offsets, source = [], routes.offsets.tolist(), routes.source
    for e in range(E):
        token = source[offsets[e]:offsets[e + 1]].long() // K
        G_y = gy[offsets[e]:offsets[e + 1]].double()
        W, Wo = wi[e].double(), wo[e].double()
        z = torch.empty(len(token), 2 * c, dtype=torch.float64, device="cuda")
        dz = torch.empty_like(z)
        for a in range(0, len(token), 8192):
            X = x[token[a:a + 8192]].double()
            z[a:a + 8192] = X @ W.T
            dz[a:a + 8192] = s(di) * (X.abs() @ W.abs().T)
        g, u, eg, eu = z[:, :c], z[:, c:], dz[:, :c], dz[:, c:]
        sg = torch.sigmoid(g)
        v, dv = g * sg, sg * (1 + g * (1 - sg))
        H = v * u
        eH = 1.2 * eg * (u.abs() + eu) + v.abs() * eu + ea * (g.abs() * u.abs())
        eH = eH + h * (H.abs() + eH)
        dH, edH = G_y @ Wo, s(do) * (G_y.abs() @ Wo.abs())
        edv = eg + ea + 4 * Q * g.abs()
        dU, dG = dH * v, dH * u * dv
        edU = edH * v.abs() + (dH.abs() + edH) * (1.2 * eg + ea * g.abs())
        edG = edH * (u * dv).abs() + (dH.abs() + edH) * ((u.abs() + eu) * edv + eu * dv.abs())
        D, eD = torch.cat([dG, dU], 1), torch.cat([edG, edU], 1)
        eD = eD + 4 * Q * D.abs()
        eD = eD + h * (D.abs() + eD)
        X = x[:, -16:][token].double()
        out.append((D, eD, X, H, eH, G_y))
    return out


def test_more_rows_than_work_groups():
    """2^22 + 5 rows of more than 2048 values: work-groups take a second row."""
    torch, lib = _setup()
    N, D, E = (1 << 22) + 5, 2051, 5
    g = torch.Generator(device="cuda").manual_seed(5)
    index = torch.randint(-1, E, (N,), generator=g, device="cuda")
    r = lib.Routes(index, E)
    M = int(r.offsets[-1])
    assert M == int((index >= 0).sum())
    x = _randn(torch, torch.bfloat16, N, D, seed=6)
    xs = r.gather(x)
    assert not xs[M:].any()
    token = r.source[:M].long()
    for a in range(0, M, 1 << 20):
        assert torch.equal(xs[a:a + (1 << 20)][: M - a], x[token[a:a + (1 << 20)]])
    w = torch.rand(N, generator=g, device="cuda")
    y, chosen = r.combine(xs, None), index >= 0
    for a in range(0, N, 1 << 20):
        assert torch.equal(y[a:a + (1 << 20)], x[a:a + (1 << 20)] * chosen[a:a + (1 << 20), None])
    del y
    gys, gw = r.combine_backward(xs, w, x)
    assert not gys[M:].any()
    for a in range(0, M, 1 << 20):
        rows = token[a:a + (1 << 20)]
        got, want = gys[a:a + (1 << 20)][: M - a], x[rows]
        assert torch.equal(got, (w[rows][:, None] * want.float()).to(torch.bfloat16))
        want = want.float().square().sum(1, dtype=torch.float64)
        assert bool(((gw[rows].double() - want).abs() <= (D / 32 + 16 + 1) * Q * want).all())
    assert not gw[~chosen].any()


def test_layer_past_32_bits():
    torch, lib = _setup()
    N, D = 70001, 32776   # 2^31 values and more
    x, gu = _randn(torch, torch.bfloat16, N, D, seed=7), _randn(torch, torch.bfloat16, N, D, seed=8)
    w, b = _randn(torch, torch.bfloat16, D, seed=9), _randn(torch, torch.bfloat16, D, seed=10)
    plan = lib.LayerNormPlan(D, dtype="bf16")
    u, stats = plan.forward(x, w, b)
    gx, gw, gb = plan.backward(x, w, stats, gu)
    rows = torch.tensor([0, 1, N // 2, 65535, 65536, N - 2, N - 1], device="cuda")
    one = [t[rows].contiguous() for t in (x, gu)]
    few = plan.backward(one[0], w, stats[:, rows].contiguous(), one[1])
    _compare(torch, lib, one[0].cpu(), w.cpu(), b.cpu(), one[1].cpu(), u[rows], stats[:, rows], (gx[rows],) + few[1:], plan.eps, "rows")
    cols = torch.tensor([0, 7, D // 2, D - 1], device="cuda")
    n = (x[:, cols].double() - stats[0].double()[:, None]) * stats[1].double()[:, None]   # with n's error as in _compare
    G = gu[:, cols].double()
    s, g = (min(N, N / 256 + 64) + 8) * Q, (D / 256 + 32) * Q
    for got, want, size in ((gw, (G * n).sum(0), (G * n).abs().sum(0)), (gb, G.sum(0), G.abs().sum(0))):
        slack = s * size + 4 * g * (G.abs() * (1 + n.abs())).sum(0) + 2.0 ** -8 * want.abs()
        assert bool(((got[cols].double() - want).abs() <= slack).all())


@pytest.mark.parametrize("N", [3, 400])
def test_two_streams_at_once(N):
    """Calls of one plan and one order that run beside each other, each with its own workspace."""
    torch, lib = _setup()
    t, E = torch.bfloat16, 6
    plan, norm = lib.ExpertsPlan(E, 192, 320, 192, dtype="bf16"), lib.LayerNormPlan(192, dtype="bf16")
    wi, wo = _randn(torch, t, E, 640, 192, scale=0.07, seed=1), _randn(torch, t, E, 192, 320, scale=0.06, seed=2)
    lw, lb = _randn(torch, t, 192, seed=3), _randn(torch, t, 192, seed=4)
    g = torch.Generator(device="cuda").manual_seed(N)
    index = torch.randint(0, E, (N, 2), generator=g, device="cuda")
    weights = torch.rand(N, 2, generator=g, device="cuda")
    inputs = [(_randn(torch, t, N, 192, seed=10 + k), _randn(torch, t, N, 192, seed=20 + k)) for k in range(6)]

    def run(x, gy, routes):
        u, stats = norm.forward(x, lw, lb)
        ys, saved = plan.forward(u, routes, wi, wo, save=True)
        y = routes.combine(ys, weights)
        gys, gw = routes.combine_backward(ys, weights, gy)
        grads = plan.backward(u, routes, wi, wo, saved, gys)
        return (y, gw) + grads + norm.backward(x, lw, stats, grads[0])

    routes = lib.Routes(index, E)
    want = [run(x, gy, routes) for x, gy in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for k, (x, gy) in enumerate(inputs):
        with torch.cuda.stream(streams[k % 2]):
            got.append(run(x, gy, routes))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
