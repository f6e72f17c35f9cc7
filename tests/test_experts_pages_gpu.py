"""The experts' blocks on arrays of odd 16-bit rows that end with a page of memory (the last expert's weights are then copied,
rows of x too), and on others with NaN behind them: the same bits."""
import pytest

from test_experts_gpu import _case, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("E,di,df,do,N", [(3, 9, 256, 8, 300), (2, 8, 257, 64, 300), (4, 7, 9, 48, 1000), (1, 9, 24, 8, 500),
                                          (2, 1023, 1024, 520, 20000), (8, 1, 1, 8, 3000), (8, 8, 3, 1, 3000)])
@pytest.mark.parametrize("kind", ["even", "one"])
def test_arrays_that_end_with_a_page(E, di, df, do, N, kind, dtype):
    torch, lib = _setup()
    index, x, wi, wo, gy = _case(torch, N, 1, E, di, df, do, dtype, kind)
    index[-1] = E - 1   # the last expert has rows
    plan = lib.ExpertsPlan(E, di, df, do, dtype=dtype)
    routes = lib.Routes(torch.from_numpy(index).cuda(), E)
    M = int(routes.offsets[E])
    outs = []
    for shift in (0, 256):
        def at_page(t):
            size = t.numel() * t.element_size()
            raw = torch.full((size + 16384,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN)
            first = (raw.data_ptr() + size + 4095) // 4096 * 4096 + 4096 - shift - size - raw.data_ptr()
            out = raw[first:first + size].view(t.dtype).view(t.shape)
            out.copy_(t)
            return out
        a = [at_page(t.cuda()) for t in (x, wi, wo, gy)]
        assert all((t.data_ptr() + t.numel() * 2) % 4096 == -shift % 4096 for t in a)
        y, saved = plan.forward(a[0], routes, a[1], a[2], save=True)
        outs.append((y[:M], saved[:M]) + plan.backward(a[0], routes, a[1], a[2], saved, a[3]))
    assert all(bool(p.isfinite().all()) and torch.equal(p, q) for p, q in zip(*outs))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("di", [1, 3, 5, 8, 12, 61, 81, 130, 257, 1089, 2050])
def test_rows_in_the_sorted_order_have_zeros_behind_them(di, dtype):
    """The rows of x that the gradients' products read, first in the workspace, in rows of a multiple of eight values."""
    torch, lib = _setup()
    N, K, E = 70, 2, 3
    index, x, wi, wo, gy = _case(torch, N, K, E, di, 16, 8, dtype, "even")
    x, wi, wo, gy = (t.cuda() for t in (x, wi, wo, gy))
    plan, routes = lib.ExpertsPlan(E, di, 16, 8, dtype=dtype), lib.Routes(torch.from_numpy(index).cuda(), E)
    _, saved = plan.forward(x, routes, wi, wo, save=True)
    ws = torch.full((lib.ffn_experts_backward_workspace_bytes(plan._h, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    plan.backward(x, routes, wi, wo, saved, gy, False, True, False, workspace=ws)
    M, ld = int(routes.offsets[E]), (di + 7) // 8 * 8
    rows = ws[:N * K * ld * x.element_size()].view(x.dtype).view(N * K, ld)[:M]
    assert torch.equal(rows[:, :di], routes.gather(x)[:M]) and bool((rows[:, di:] == 0).all())
