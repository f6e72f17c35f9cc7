"""The layer norm on several rows a worker in every form of its kernels, against its definition in 64 bits, with the
tolerances derived in test_layer_gpu."""
import pytest

from test_layer_gpu import _compare, _inputs, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,D", [(1025, 1000), (600, 1024), (530, 2500), (300, 4096), (270, 8000), (260, 12001), (258, 16384)])
def test_several_rows_a_worker(N, D, dtype):
    torch, lib = _setup()
    x, w, b, gu = _inputs(torch, N, D, dtype, seed=D)
    plan = lib.LayerNormPlan(D, dtype=dtype)
    dx, dw, db, dgu = (t.cuda() for t in (x, w, b, gu))
    u, stats = plan.forward(dx, dw, db)
    _compare(torch, lib, x, w, b, gu, u, stats.cpu(), plan.backward(dx, dw, stats, dgu), plan.eps, "%d x %d" % (N, D))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [6, 64, 1000, 1089, 4096, 9001, 20000])
def test_rows_beyond_the_range_of_squares(D, dtype):
    """Values whose squares are infinite in 32 bits (1e20: the mean's correction squared is not, 1e30: it is): r is 0 and u is
    b, and other rows keep their bits.  Rows with NaN or infinities: both statistics are NaN."""
    torch, lib = _setup()
    x, w, b, _ = (t.cuda() for t in _inputs(torch, 40, D, dtype))
    plan = lib.LayerNormPlan(D, dtype=dtype)
    u, stats = plan.forward(x, w, b)
    bad = x.clone()
    bad[3], bad[11] = x[3] * 1e20, x[11] * 1e30
    bad[20, D // 2], bad[31, D - 1], bad[32, 0] = float("nan"), float("inf"), -float("inf")
    u2, stats2 = plan.forward(bad, w, b)
    keep = [i for i in range(40) if i not in (3, 11, 20, 31, 32)]
    assert torch.equal(u2[keep], u[keep]) and torch.equal(stats2[:, keep], stats[:, keep])
    assert not stats2[1, [3, 11]].any() and stats2[0, [3, 11]].isfinite().all()
    assert torch.equal(u2[3], b) and torch.equal(u2[11], b)
    assert u2[[20, 31, 32]].isnan().all() and stats2[:, [20, 31, 32]].isnan().all()
