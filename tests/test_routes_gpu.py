"""Rows sorted by expert and brought back (include/experts.h) on the GPU against their definitions.

The order is whole numbers and has to be equal.  Sums are held in 32 bits (q = 2^-24 a step): a row of K choices is K
products added in line, off by at most (K + 1) q of the sum of magnitudes, then rounded once by half a step h of its type;
the product of two rows of D values takes at most D / 32 + 16 additions in line.
"""
import numpy as np
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


def _order(index, experts):
    """(place, source, offsets) of a numpy array [N, K], by a loop over experts."""
    flat = index.reshape(-1)
    source = np.concatenate([np.nonzero(flat == e)[0] for e in range(experts)])
    offsets = np.concatenate([[0], np.cumsum([(flat == e).sum() for e in range(experts)])])
    place = np.full(flat.size, -1)
    place[source] = np.arange(source.size)
    return place.reshape(index.shape), np.concatenate([source, np.full(flat.size - source.size, -1)]), offsets


def _index(N, K, E, kind, seed=0):
    r = np.random.default_rng(seed + N + 7 * K + 31 * E)
    if kind == "one":
        return np.full((N, K), E - 1)
    if kind == "none":
        return np.full((N, K), -1)
    index = r.integers(0, E, (N, K))   # the same expert twice among them
    if kind == "some":
        index = np.where(r.random((N, K)) < 0.4, r.choice([-1, E, E + 5, -2 ** 31, 2 ** 31 - 1], (N, K)), index)
    if kind == "skewed":
        index = np.minimum(index, r.integers(0, E, (N, K)) // 3)
    return index


@pytest.mark.parametrize("N,K,E", [(1, 1, 1), (1, 2, 8), (3, 3, 2), (64, 1, 5), (65, 2, 64), (100, 8, 65), (1000, 3, 7),
                                   (8192, 1, 16), (8193, 1, 3), (5000, 2, 1024), (20000, 4, 100), (300000, 1, 255),
                                   (7, 1024, 1000)])
@pytest.mark.parametrize("kind", ["even", "some", "skewed", "one", "none"])
def test_order(N, K, E, kind):
    torch, lib = _setup()
    index = _index(N, K, E, kind)
    want = _order(index, E)
    for dtype in (torch.int64, torch.int32):
        r = lib.Routes(torch.from_numpy(index).to(dtype).cuda(), E)
        for got, w in zip((r.place, r.source, r.offsets), want):
            assert got.dtype == torch.int32 and np.array_equal(got.cpu().numpy(), w)
    if K == 1:
        r = lib.Routes(torch.from_numpy(index[:, 0].copy()).cuda(), E)
        assert r.place.shape == (N,) and np.array_equal(r.place.cpu().numpy(), want[0][:, 0])


def test_choices_of_64_bits_are_not_cut_off():
    torch, lib = _setup()
    index = torch.tensor([[2 ** 32 + 1, 1], [-2 ** 40, 0], [2 ** 62, -1]], device="cuda")
    r = lib.Routes(index, 4)
    assert r.place.tolist() == [[-1, 1], [-1, 0], [-1, -1]] and r.offsets.tolist() == [0, 1, 2, 2, 2]
    assert r.source.tolist() == [3, 1, -1, -1, -1, -1]


def _case(torch, N, K, E, D, dtype, kind, seed=0):
    index = _index(N, K, E, kind, seed)
    g = torch.Generator().manual_seed(seed)
    t = _dt(torch, dtype)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).to(t)
    return index, r(N, D), r(N * K, D), torch.rand(N, K, generator=g), r(N * K, D), r(N, D)


def _close(torch, got, want, slack):
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -130
    h = torch.finfo(got.dtype).eps / 2
    assert bool(((got.double().cpu() - want).abs() <= h * want.abs() + slack + tiny).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,K,E,D", [(1, 2, 8, 4096), (1, 1, 1, 1), (5, 3, 4, 7), (64, 2, 8, 64), (333, 4, 5, 100),
                                     (1001, 1, 6, 33), (40, 6, 9, 1089), (4200, 2, 16, 24), (9, 2, 3, 9000),
                                     (2, 20, 30, 130), (5000, 3, 4, 8)])
@pytest.mark.parametrize("kind", ["even", "some", "none"])
def test_rows_there_and_back(N, K, E, D, dtype, kind):
    torch, lib = _setup()
    index, x, ys, w, gxs, gy = _case(torch, N, K, E, D, dtype, kind)
    place, source, offsets = _order(index, E)
    M = offsets[-1]
    ys[M:], gxs[M:] = float("nan"), float("nan")       # rows behind the last are not read
    w[torch.from_numpy(place < 0)] = float("nan")      # nor weights of no expert
    r = lib.Routes(torch.from_numpy(index).cuda(), E)
    dx, dys, dw, dgxs, dgy = (t.cuda() for t in (x, ys, w, gxs, gy))
    xs = r.gather(dx).cpu()
    token = torch.from_numpy(source[:M] // K)
    assert torch.equal(xs[:M], x[token]) and not xs[M:].any()

    slot = torch.from_numpy(source[:M])
    w64, ys64 = w.double().reshape(-1)[slot][:, None], ys.double()[:M]
    zero = torch.zeros(N, D, dtype=torch.float64)
    add = lambda v: zero.index_add(0, token, v)
    _close(torch, r.combine(dys, dw), add(w64 * ys64), (K + 1) * Q * add((w64 * ys64).abs()))
    _close(torch, r.combine(dys), add(ys64), K * Q * add(ys64.abs()))
    _close(torch, r.gather_backward(dgxs), add(gxs.double()[:M]), K * Q * add(gxs.double()[:M].abs()))
    gys, gw = r.combine_backward(dys, dw, dgy)
    g64 = gy.double()[token]
    _close(torch, gys[:M], w64 * g64, Q * (w64 * g64).abs())
    assert not gys[M:].any()
    want = torch.zeros(N * K, dtype=torch.float64)
    size = want.clone()
    want[slot], size[slot] = (g64 * ys64).sum(1), (g64 * ys64).abs().sum(1)
    _close(torch, gw, want.reshape(N, K), ((D / 32 + 16) * Q * size).reshape(N, K))
    assert gw.dtype == torch.float32 and not gw.cpu()[torch.from_numpy(place < 0)].any()
    a, b = r.combine_backward(None, dw, dgy, need_weights=False)
    assert b is None and torch.equal(a, gys)
    a, b = r.combine_backward(dys, None, dgy, need_ys=False)
    assert a is None and torch.equal(b, gw)
    ones = r.combine_backward(dys, None, dgy)[0]
    assert torch.equal(ones[:M].cpu(), gy[token])
    assert r.combine_backward(None, None, dgy, False, False) == (None, None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [5, 80, 301])
def test_strided_rows_and_other_stream(D, dtype):
    torch, lib = _setup()
    N, K, E = 50, 2, 6
    index, x, ys, w, gxs, gy = _case(torch, N, K, E, D, dtype, "some")
    side = torch.cuda.Stream()
    r = lib.Routes(torch.from_numpy(index).cuda(), E)
    x, ys, w, gy = (t.cuda() for t in (x, ys, w, gy))
    wide = torch.full((N, D + 7), float("nan"), dtype=x.dtype, device="cuda")
    gwide, out = wide.clone(), wide.clone()
    wide[:, 3:3 + D], gwide[:, 1:1 + D] = x, gy
    xs, y, gb = r.gather(x), r.combine(ys, w), r.combine_backward(ys, w, gy)
    assert torch.equal(r.gather(wide[:, 3:3 + D]), xs)
    r.combine(ys, w, out=out[:, 2:2 + D])
    assert torch.equal(out[:, 2:2 + D], y) and out[:, :2].isnan().all() and out[:, 2 + D:].isnan().all()
    assert all(torch.equal(a, b) for a, b in zip(r.combine_backward(ys, w, gwide[:, 1:1 + D]), gb))
    side.wait_stream(torch.cuda.current_stream())
    r2 = lib.Routes(torch.from_numpy(index).cuda(), E, stream=side)
    torch.cuda.current_stream().wait_stream(side)   # (index was copied on the current stream, which it waited for)
    side.wait_stream(torch.cuda.current_stream())
    xs2, y2 = r2.gather(x, stream=side), r2.combine(ys, w, stream=side)
    gb2 = r2.combine_backward(ys, w, gy, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(xs2, xs) and torch.equal(y2, y) and all(torch.equal(a, b) for a, b in zip(gb2, gb))


def test_no_rows():
    torch, lib = _setup()
    r = lib.Routes(torch.empty(0, 3, dtype=torch.int64, device="cuda"), 5)
    assert r.offsets.tolist() == [0] * 6 and r.source.shape == (0,) and r.place.shape == (0, 3)
    x = torch.empty(0, 16, device="cuda")
    assert r.gather(x).shape == (0, 16) and r.combine(x, torch.empty(0, 3, device="cuda")).shape == (0, 16)
    gys, gw = r.combine_backward(x, torch.empty(0, 3, device="cuda"), x)
    assert gys.shape == (0, 16) and gw.shape == (0, 3)


def test_infinities_stay_in_their_rows():
    """An infinite row of one expert, and an infinite weight, reach the rows that chose them and no others."""
    torch, lib = _setup()
    index, x, ys, w, _, gy = _case(torch, 60, 2, 5, 72, "fp32", "even")
    r = lib.Routes(torch.from_numpy(index).cuda(), 5)
    want = r.combine(ys.cuda(), w.cuda()).cpu()
    ys2, w2 = ys.clone(), w.clone()
    ys2[9], w2[11, 1] = float("inf"), float("inf")
    hit = int(r.source[9]) // 2
    got = r.combine(ys2.cuda(), w2.cuda()).cpu()
    keep = [n for n in range(60) if n not in (hit, 11)]
    assert torch.equal(got[keep], want[keep]) and not got[hit].isfinite().any() and not got[11].isfinite().any()


def test_captured_and_replayed():
    """Sorting, gathering and both gradients in one graph, replayed on new choices with eager calls between."""
    torch, lib = _setup()
    for N, K, E, D in ((3, 2, 4, 64), (6000, 2, 20, 40)):
        sets = [_case(torch, N, K, E, D, "bf16", ("even", "some", "one", "none")[s], s) for s in range(4)]
        sets = [[torch.from_numpy(s[0]).cuda()] + [t.cuda() for t in s[1:]] for s in sets]
        args = [t.clone() for t in sets[0]]

        def step(index, x, ys, w, gxs, gy):
            r = lib.Routes(index, E)
            return (r.place, r.source, r.offsets, r.gather(x), r.combine(ys, w), r.gather_backward(gxs)) + \
                r.combine_backward(ys, w, gy)

        step(*args)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*args)
        for s in sets + sets[:2]:
            for to, fr in zip(args, s):
                to.copy_(fr)
            graph.replay()
            want = step(*s)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    torch, lib = _setup()
    index = torch.zeros(6, 2, dtype=torch.int64, device="cuda")
    for bad in (index.cpu(), index.float(), index.to(torch.int16), index.t(), index[None], index[:, :0]):
        with pytest.raises(ValueError):
            lib.Routes(bad, 3)
    for experts in (0, -1, 1025):
        with pytest.raises(ValueError):
            lib.Routes(index, experts)
    r = lib.Routes(index, 3)
    x, ys, w = (torch.zeros(n, 8, device="cuda") for n in (6, 12, 6))
    w = torch.zeros(6, 2, device="cuda")
    for bad in (x[:5], x.double(), x.cpu(), x[:, :0], x.t()):
        with pytest.raises(ValueError):
            r.gather(bad)
    for bad in (ys[:11], ys.double(), ys.cpu(), torch.zeros(12, 16, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            r.combine(bad, w)
    for bad in (w[:5], w.half(), w.reshape(-1), w.t().contiguous().t()):
        with pytest.raises(ValueError):
            r.combine(ys, bad)
        with pytest.raises(ValueError):
            r.combine_backward(ys, bad, x)
    with pytest.raises(ValueError):
        r.combine_backward(None, w, x)
    with pytest.raises(ValueError):
        r.combine_backward(ys.half(), w, x)
    with pytest.raises(ValueError):
        r.gather(x, out=torch.empty(12, 7, device="cuda"))
    with pytest.raises(lib.CgtpError):
        r.gather(ys[:6], out=ys)
