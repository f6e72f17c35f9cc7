"""A network layer around the full Clebsch-Gordan tensor product, trained and served.

Per-pair scalars (a radial basis, species features) pass through one residual
feed-forward sublayer and a second block that gives one weight per (channel,
path); the weights scale the paths of the channel-wise product of node features
with the pairs' spherical harmonics:

    u  = N(s; w_pre)                                 norm before the block
    h  = Block1(u)                                   gated feed-forward block
    t  = s + scale * gate * drop(N(h; w_post)),  v = N(t; w_next)
    p  = Block2(v)                                   [pairs, channels * paths]
    z  = product of x1 [pairs, channels, (L+1)^2] and x2 [pairs, (L+1)^2], path weights p

Training fits p to given weights by gradient descent through every operator.

    python examples/path_weights.py [--pairs N] [--steps K]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2602_21466_amd as cg  # noqa: E402


class PathWeights:
    """The sublayer and the block that makes the weights; parameters are plain tensors."""

    def __init__(self, width, hidden, outputs, dtype="fp32", dropout=0.1, seed=0):
        tdt = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5
        ones = lambda: torch.ones(width, device="cuda")
        self.block1 = cg.FfnPlan(width, hidden, width, dtype=dtype)
        self.block2 = cg.FfnPlan(width, hidden, outputs, dtype=dtype)
        self.train_norm = cg.NormPlan(width, dtype=dtype, dropout=dropout)
        self.norm = cg.NormPlan(width, dtype=dtype)
        p = {"pre": ones(), "post": ones(), "next": ones(), "scale": ones() * 0.5,
             "in1": rand(2 * hidden, width), "out1": rand(width, hidden),
             "in2": rand(2 * hidden, width), "out2": rand(outputs, hidden)}
        self.p = {k: v.to(tdt) for k, v in p.items()}

    def serve(self, s, gate):
        p = self.p
        u, _ = self.norm.forward(s, p["pre"])
        h = self.block1.forward(u, p["in1"], p["out1"])
        _, v, _ = self.norm.residual(s, h, p["post"], gate=gate, scale=p["scale"], w_next=p["next"])
        return self.block2.forward(v, p["in2"], p["out2"])

    def train_step(self, s, gate, target, rate, step):
        """One step of gradient descent on the mean square distance to target; returns it before the step."""
        p, norm, rng = self.p, self.train_norm, {"seed": 1234, "offset": step}
        u, rstd = norm.forward(s, p["pre"])
        h, saved1 = self.block1.forward(u, p["in1"], p["out1"], save=True)
        join = {"gate": gate, "scale": p["scale"], "w_next": p["next"], **rng}
        t, v, stats = norm.residual(s, h, p["post"], **join)
        out, saved2 = self.block2.forward(v, p["in2"], p["out2"], save=True)

        diff = out.float() - target.float()
        grad = (diff * (2.0 / diff.numel()) * 2.0 ** 12).to(out.dtype)   # scaled: small gradients keep their bits in fp16
        g = {}
        gv, g["in2"], g["out2"] = self.block2.backward(v, p["in2"], p["out2"], saved2, grad)
        _, gh, g["post"], _, g["scale"], g["next"] = norm.residual_backward(h, t, p["post"], stats, None, gv, **join)
        gu, g["in1"], g["out1"] = self.block1.backward(u, p["in1"], p["out1"], saved1, gh)
        _, g["pre"] = norm.backward(s, p["pre"], rstd, gu, need_x=False)
        for k, v in g.items():
            p[k].sub_((v.float() * (rate / 2.0 ** 12)).to(p[k].dtype))
        return float(diff.square().mean())


def main(pairs=1024, steps=30, L=4, channels=4, width=64, hidden=256, dtype="fp32"):
    paths = cg.cgtp_num_paths(L)
    g = torch.Generator(device="cuda").manual_seed(7)
    net = PathWeights(width, hidden, channels * paths, dtype=dtype)
    tdt = net.p["pre"].dtype
    s = torch.randn(pairs, width, generator=g, device="cuda").to(tdt)
    gate = torch.randn(pairs, width, generator=g, device="cuda").sigmoid().to(tdt)
    target = torch.tanh(s.float() @ torch.randn(width, channels * paths, generator=g, device="cuda") * width ** -0.5)
    losses = [net.train_step(s, gate, target, rate=30.0, step=k) for k in range(steps)]
    weights = net.serve(s, gate).float().reshape(pairs, channels, paths)
    x1 = torch.randn(pairs, channels, (L + 1) ** 2, generator=g, device="cuda")
    x2 = torch.randn(pairs, (L + 1) ** 2, generator=g, device="cuda")
    z = cg.Plan(L).forward_weighted(x1, x2, weights)
    torch.cuda.synchronize()
    return losses, weights, z


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--pairs", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", default="fp32", choices=("fp32", "bf16", "fp16"))
    a = ap.parse_args()
    losses, weights, z = main(a.pairs, a.steps, dtype=a.dtype)
    print("loss %.4f -> %.4f over %d steps; weights %s, products %s" %
          (losses[0], losses[-1], len(losses), list(weights.shape), list(z.shape)))
