"""The feed-forward sublayer where single values, views and the division of rows tell: bounds that hold for every value
and not in the mean of many, arrays that lie in one another's gaps or in place of one another, and plans that differ in
what a call does not read."""
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
