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
