"""A residual mixture through the layer norm, the routes and the experts' blocks in fp32, with all its gradients, against torch
in 64 bits by norms.

Tolerance.  A sum of K products over bf16 parts leaves out 2^-25.5 of each product in the root mean square, of either sign, and
its K / 16 + 40 additions or fewer round the sum so far by 2^-24 at the most, 2^-25 and less in the root mean square: for the
sizes here (K up to 300) at most (2^-51 + 59 * 2^-50)^(1/2) < 2^-22 of a result's norm.  The longest way through the operators passes
the norm (two sums), two products forward, the weighted sum, its gradient, three products and the sum over choices backward and
the norm's gradient (two sums): twelve, added as if they all had one sign: 12 * 2^-22.
"""
import numpy as np
import pytest

from test_experts_gpu import _case, _mixture, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,E,D,F", [(120, 2, 6, 56, 88), (9, 3, 4, 64, 96), (700, 1, 3, 75, 150), (300, 4, 8, 40, 130)])
def test_mixture_and_its_gradients_by_norms(N, K, E, D, F):
    torch, lib = _setup()
    index, x, wi, wo, _ = _case(torch, N, K, E, D, F, D, "fp32", "some", seed=11)
    g = torch.Generator().manual_seed(4)
    lw, lb, w, gy = (torch.randn(s, generator=g) for s in ((D,), (D,), (N, K), (N, D)))
    norm, plan = lib.LayerNormPlan(D), lib.ExpertsPlan(E, D, F, D)
    got = _mixture(lib, norm, plan, *(t.cuda() for t in (x, lw, lb, torch.from_numpy(index), w, wi, wo, gy)))
    leaves = [t.double().requires_grad_(True) for t in (x, lw, lb, w, wi, wo)]
    x6, lw6, lb6, w6, wi6, wo6 = leaves
    c = x6 - x6.mean(1, keepdim=True)
    u = c / (c.square().mean(1, keepdim=True) + norm.eps).sqrt() * lw6 + lb6
    t = x6
    for e in range(E):
        rows, k = np.nonzero(index == e)
        z = u[rows] @ wi6[e].T
        y = (torch.nn.functional.silu(z[:, :F]) * z[:, F:]) @ wo6[e].T
        t = t.index_add(0, torch.from_numpy(rows), w6[rows, k][:, None] * y)
    want = [t.detach()] + list(torch.autograd.grad(t, leaves, gy.double()))
    for name, a, b in zip(("t", "gx", "glw", "glb", "gweights", "gw_in", "gw_out"), got, want):
        assert float((a.double().cpu() - b).norm()) <= 12 * 2.0 ** -22 * float(b.norm()), name
