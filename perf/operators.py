"""Cases of use of the feed-forward sublayer's operators, for timing and checking them.

Each case is one pass of a user's program through one operator: the gated
feed-forward block (serving and training), the norms before and after a block
fused with its gate and residual scale, and counter-based dropout.  With `own`
false a pass is the operator's plain form: elementary torch operations in 32
bits, rounded once at the end.  With `own` true it is the library's calls.

    listed()            the cases, dicts of plain values
    draw(rng)           one more case of the same ranges
    prepare(case, s)    inputs (and the plan) on the GPU, from the seed alone
    run(state)          one pass; returns its outputs
    work(case)          bytes and flops a pass cannot do without
    exact(case, s)      what run() returns, in 64 bits from the definitions
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6

# op "ffn":      Y = (act(X Wg^T) * (X Wu^T)) Wo^T; train adds the gradients of X and of both weights
# op "before":   u = N(x; w), the root-mean-square norm of each row; train adds its gradients
# op "after":    y = x + scale * gate * drop(N(h; w)) and u = N(y; w_next); train adds all their gradients
# op "dropout":  y = drop(x); train adds the gradient


def listed():
    return [
        # one token's features through a wide block: the weights are all there is to read
        {"name": "ffn_serve_bf16_1x2048x8192", "op": "ffn", "train": False, "dtype": "bf16", "rows": 1, "d_in": 2048,
         "d_ff": 8192, "d_out": 2048, "act": "silu"},
        # a small batch served together
        {"name": "ffn_serve_bf16_24x4096x16384", "op": "ffn", "train": False, "dtype": "bf16", "rows": 24,
         "d_in": 4096, "d_ff": 16384, "d_out": 4096, "act": "silu"},
        # path weights of 64 pairs at L = 8 (81 features in, 489 paths out): the smallest call, odd sizes
        {"name": "ffn_serve_fp32_64x81x324x489", "op": "ffn", "train": False, "dtype": "fp32", "rows": 64, "d_in": 81,
         "d_ff": 324, "d_out": 489, "act": "silu"},
        # a ragged batch of L = 32 feature rows (1089 values), every size odd or unaligned
        {"name": "ffn_serve_fp16_1001x1089x2903", "op": "ffn", "train": False, "dtype": "fp16", "rows": 1001,
         "d_in": 1089, "d_ff": 2903, "d_out": 1089, "act": "gelu"},
        # training the block that makes the path weights of 8192 pairs at L = 16 (3281 paths)
        {"name": "ffn_train_fp32_8192x128x512x3281", "op": "ffn", "train": True, "dtype": "fp32", "rows": 8192,
         "d_in": 128, "d_ff": 512, "d_out": 3281, "act": "silu"},
        # a training step of a large block: the most arithmetic
        {"name": "ffn_train_bf16_8192x4096x16384", "op": "ffn", "train": True, "dtype": "bf16", "rows": 8192,
         "d_in": 4096, "d_ff": 16384, "d_out": 4096, "act": "silu"},
        # the join of one served row: launch and latency
        {"name": "after_serve_bf16_1x4096", "op": "after", "train": False, "dtype": "bf16", "rows": 1, "width": 4096,
         "rows_per_gate": 1, "p": 0.0},
        # training, the norm before a block on L = 16 feature rows of 512 pairs x 16 channels
        {"name": "before_train_fp32_8192x289", "op": "before", "train": True, "dtype": "fp32", "rows": 8192,
         "width": 289},
        # training, ragged odd rows, one gate row a feature row
        {"name": "after_train_fp16_4001x1089", "op": "after", "train": True, "dtype": "fp16", "rows": 4001,
         "width": 1089, "rows_per_gate": 1, "p": 0.0},
        # training, a long batch whose sequences of 512 rows share their gate, with dropout
        {"name": "after_train_bf16_16384x4096", "op": "after", "train": True, "dtype": "bf16", "rows": 16384,
         "width": 4096, "rows_per_gate": 512, "p": 0.1},
        # dropout and its gradient on the same odd feature rows, and on a block's wide rows
        {"name": "dropout_train_fp32_8192x289", "op": "dropout", "train": True, "dtype": "fp32", "rows": 8192,
         "width": 289, "p": 0.25},
        {"name": "dropout_train_bf16_8192x16384", "op": "dropout", "train": True, "dtype": "bf16", "rows": 8192,
         "width": 16384, "p": 0.1},
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; half of the larger ones are multiples of 8."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = max(lo, min(hi, n))
    return n // 8 * 8 if n >= 64 and rng.random() < 0.5 else n


def draw(rng):
    while True:
        c = _draw(rng)
        if 3072 not in c.values():  # the one size that no case has
            return c


def _draw(rng):
    op = rng.choice(["ffn", "ffn", "before", "after", "dropout"])
    c = {"op": op, "train": rng.random() < 0.6, "dtype": rng.choice(["fp32", "bf16", "fp16"])}
    if op == "ffn":
        c["d_in"], c["d_ff"] = _log(rng, 64, 4096), _log(rng, 128, 16384)
        c["d_out"] = c["d_in"] if rng.random() < 0.5 else _log(rng, 64, 4096)
        c["rows"] = _log(rng, 1, 16384)
        # within the largest listed case; 32-bit blocks are those of path weights, a sixteenth of its work
        most = 9e12 if c["dtype"] != "fp32" else 6e11
        rows = int(most / (6 * c["d_ff"] * (2 * c["d_in"] + c["d_out"])))
        c["rows"] = max(1, min(c["rows"], rows))
        c["act"] = rng.choice(["silu", "gelu", "relu"])
        return c
    c["width"] = _log(rng, 16, 16384)
    c["rows"] = max(1, min(_log(rng, 1, 65536), 16384 * 4096 // c["width"]))
    if op == "after":
        c["rows_per_gate"] = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
        c["p"] = rng.choice([0.0, 0.1, 0.25])
    if op == "dropout":
        c["p"] = rng.choice([0.1, 0.25, 0.5])
    return c


def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale + mean).to(dt)

    s = {"case": case, "seed": seed, "offset": seed // 7}
    n = case["rows"]
    if case["op"] == "ffn":
        di, df, do = case["d_in"], case["d_ff"], case["d_out"]
        s["x"] = normal(n, di)  # features as a norm leaves them
        s["w_in"] = normal(2 * df, di, scale=di ** -0.5)
        s["w_out"] = normal(do, df, scale=df ** -0.5)
        if case["train"]:
            s["gy"] = normal(n, do)
        if own:
            import paper_2602_21466_amd as lib
            s["plan"] = lib.FfnPlan(di, df, do, dtype=case["dtype"], activation=case["act"])
        return s
    d = case["width"]
    s["x"] = normal(n, d)
    if case["op"] != "dropout":
        s["w"] = normal(d, scale=0.1, mean=1.0)
    if case["op"] == "after":
        s["h"] = normal(n, d, scale=0.3)
        s["gate"] = normal(-(-n // case["rows_per_gate"]), d)
        s["scale"] = normal(d, scale=0.1, mean=0.5)
        s["w_next"] = normal(d, scale=0.1, mean=1.0)
    if case["train"]:
        s["gu"] = normal(n, d)
        if case["op"] == "after":
            s["gy"] = normal(n, d)
    if own and case["op"] != "dropout":
        import paper_2602_21466_amd as lib
        s["plan"] = lib.NormPlan(d, dtype=case["dtype"], eps=EPS, rows_per_gate=case.get("rows_per_gate", 1),
                                 dropout=case.get("p", 0.0))
    return s


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2602_21466_amd as lib
    c, train = s["case"], s["case"]["train"]
    if c["op"] == "ffn":
        if not train:
            return s["plan"].forward(s["x"], s["w_in"], s["w_out"])
        y, saved = s["plan"].forward(s["x"], s["w_in"], s["w_out"], save=True)
        return (y,) + tuple(s["plan"].backward(s["x"], s["w_in"], s["w_out"], saved, s["gy"]))
    if c["op"] == "before":
        u, rstd = s["plan"].forward(s["x"], s["w"])
        return (u,) + tuple(s["plan"].backward(s["x"], s["w"], rstd, s["gu"])) if train else u
    if c["op"] == "after":
        rng = {"seed": s["seed"], "offset": s["offset"]}
        y, u, stats = s["plan"].residual(s["x"], s["h"], s["w"], gate=s["gate"], scale=s["scale"],
                                         w_next=s["w_next"], **rng)
        if not train:
            return y, u
        return (y, u) + tuple(s["plan"].residual_backward(s["h"], y, s["w"], stats, s["gy"], s["gu"], gate=s["gate"],
                                                          scale=s["scale"], w_next=s["w_next"], **rng))
    y = lib.dropout(s["x"], c["p"], seed=s["seed"], offset=s["offset"])
    return (y, lib.dropout(s["gu"], c["p"], seed=s["seed"], offset=s["offset"])) if train else y


# ---------------------------------------------------------------- the plain form

def _act(g, name):
    """act(g) and its derivative."""
    if name == "silu":
        e = 1.0 / (1.0 + torch.exp(-g))
        return g * e, e * (1.0 + g * (1.0 - e))
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    pos = (g > 0).to(g.dtype)
    return g * pos, pos


def _keep(rows, width, p, seed, offset, device):
    """1 / (1 - p) where a value is kept and 0 where it is dropped (32 bits), from Philox 4x32-10: counter
    (column / 8, row, offset), key seed; column c takes the 16 bits from 16 (c % 8) on of the block."""
    t = int(p * 65536.0 + 0.5)
    low = 0xFFFFFFFF
    blocks = -(-width // 8)
    c0 = torch.arange(blocks, device=device, dtype=torch.int64).expand(rows, blocks)
    c1 = torch.arange(rows, device=device, dtype=torch.int64)[:, None].expand(rows, blocks)
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, (offset >> 32) & low)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # products wrap at 64 bits; their halves are exact
        c0, c1, c2, c3 = (b >> 32) & low ^ c1 ^ k0, b & low, (a >> 32) & low ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 2)
    bits = bits.reshape(rows, blocks * 8)[:, :width]
    return (bits >= t).to(torch.float32) * (65536.0 / (65536 - t))


def _norm(v, w):
    r = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r * w, r


def _norm_grad(gu, v, w, r):
    """Gradients of N(v; w) with respect to v and w."""
    n, a = v * r, gu * w
    return r * (a - n * (a * n).mean(1, keepdim=True)), (gu * n).sum(0)


def _run_plain(s):
    c, train = s["case"], s["case"]["train"]
    dt = DTYPES[c["dtype"]]
    f = {k: v.float() for k, v in s.items() if torch.is_tensor(v)}
    if c["op"] == "ffn":
        df = c["d_ff"]
        gate, up = f["x"] @ f["w_in"][:df].T, f["x"] @ f["w_in"][df:].T
        a, da = _act(gate, c["act"])
        h = a * up
        y = h @ f["w_out"].T
        if not train:
            return y.to(dt)
        dh = f["gy"] @ f["w_out"]
        d = torch.cat([dh * up * da, dh * a], 1)
        return y.to(dt), (d @ f["w_in"]).to(dt), (d.T @ f["x"]).to(dt), (f["gy"].T @ h).to(dt)
    if c["op"] == "before":
        u, r = _norm(f["x"], f["w"])
        if not train:
            return u.to(dt)
        return (u.to(dt),) + tuple(v.to(dt) for v in _norm_grad(f["gu"], f["x"], f["w"], r))
    if c["op"] == "after":
        n, rpg = c["rows"], c["rows_per_gate"]
        g = f["gate"].repeat_interleave(rpg, 0)[:n]
        v, r = _norm(f["h"], f["w"])
        if c["p"] > 0:
            m = _keep(n, c["width"], c["p"], s["seed"], s["offset"], f["x"].device)
            v = v * m
        y = f["x"] + f["scale"] * g * v
        u, rn = _norm(y, f["w_next"])
        if not train:
            return y.to(dt), u.to(dt)
        gx, gwn = _norm_grad(f["gu"], y, f["w_next"], rn)
        gx = gx + f["gy"]
        groups = torch.arange(n, device=gx.device) // rpg
        ggate = torch.zeros_like(f["gate"]).index_add_(0, groups, gx * f["scale"] * v)
        gscale = (gx * g * v).sum(0)
        gv = gx * f["scale"] * g
        gh, gw = _norm_grad(gv * m if c["p"] > 0 else gv, f["h"], f["w"], r)
        return tuple(v.to(dt) for v in (y, u, gx, gh, gw, ggate, gscale, gwn))
    m = _keep(c["rows"], c["width"], c["p"], s["seed"], s["offset"], f["x"].device)
    y = (f["x"] * m).to(dt)
    return (y, (f["gu"] * m).to(dt)) if train else y


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    e, n = SIZE[case["dtype"]], case["rows"]
    if case["op"] == "ffn":
        di, df, do = case["d_in"], case["d_ff"], case["d_out"]
        flops = 2.0 * n * df * (2 * di + do)
        values = n * (di + do) + df * (2 * di + do)
        if case["train"]:
            # forward, and twice its products backward; x, y, dy, dx once each, both weights and their gradients
            return {"flops": 3 * flops, "bytes": e * (2 * n * (di + do) + 2 * df * (2 * di + do))}
        return {"flops": flops, "bytes": e * values}
    d = case["width"]
    if case["op"] == "before":
        # x in, u out; gradients: gu in, gx out (x is read once in all), the weight and its gradient
        return {"flops": n * d * (13.0 if case["train"] else 4.0),
                "bytes": e * ((4 * n + 2) * d if case["train"] else (2 * n + 1) * d)}
    if case["op"] == "after":
        gates = -(-n // case["rows_per_gate"])
        values = (4 * n + gates + 3) * d
        if case["train"]:
            # x, h, y, u and gy, gu, gx, gh; the gate, three rows of weights, and their gradients
            return {"flops": 40.0 * n * d, "bytes": e * ((8 * n + 2 * gates + 6) * d)}
        return {"flops": 12.0 * n * d, "bytes": e * values}
    return {"flops": n * d * 2.0, "bytes": e * n * d * (4 if case["train"] else 2)}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_keep(rows, width, p, seed, offset):
    """The dropout factors in 64 bits, by unsigned 64-bit host arithmetic."""
    t = math.floor(p * 65536.0 + 0.5)
    u32, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    blocks = (width + 7) // 8
    col, row = np.meshgrid(np.arange(blocks, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    c = [col.ravel(), row.ravel(), np.full(rows * blocks, offset & 0xFFFFFFFF, dtype=np.uint64),
         np.full(rows * blocks, (offset >> 32) & 0xFFFFFFFF, dtype=np.uint64)]
    for i in range(10):
        k0 = np.uint64(((seed & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((seed >> 32 & 0xFFFFFFFF) + i * 0xBB67AE85) & 0xFFFFFFFF)
        x, z = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(z >> sh) ^ c[1] ^ k0, z & u32, (x >> sh) ^ c[3] ^ k1, x & u32]
    words = np.stack(c, 1).astype("<u4").view("<u2").reshape(rows, blocks * 8)[:, :width]
    return torch.from_numpy((words >= t).astype(np.float64) * (65536.0 / (65536.0 - t))).cuda()


def _rms(v, w):
    return w * v / (v.square().mean(-1, keepdim=True) + EPS).sqrt()


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    f = {k: v.double().requires_grad_(c["train"]) for k, v in s.items() if torch.is_tensor(v)}
    if c["op"] == "ffn":
        z = f["x"] @ f["w_in"].T
        a, b = z[:, :c["d_ff"]], z[:, c["d_ff"]:]
        a = {"silu": lambda v: v * torch.sigmoid(v), "relu": lambda v: v.clamp_min(0.0),
             "gelu": lambda v: v * torch.special.ndtr(v)}[c["act"]](a)
        y = (a * b) @ f["w_out"].T
        if not c["train"]:
            return y
        return (y.detach(),) + torch.autograd.grad(y, (f["x"], f["w_in"], f["w_out"]), f["gy"])
    if c["op"] == "before":
        u = _rms(f["x"], f["w"])
        return (u.detach(),) + torch.autograd.grad(u, (f["x"], f["w"]), f["gu"]) if c["train"] else u
    keep = None
    if c["p"] > 0:
        keep = _exact_keep(c["rows"], c["width"], c["p"], s["seed"], s["offset"])
    if c["op"] == "dropout":
        y = f["x"].detach() * keep
        return (y, f["gu"].detach() * keep) if c["train"] else y
    group = torch.arange(c["rows"], device="cuda") // c["rows_per_gate"]
    v = _rms(f["h"], f["w"])
    v = v if keep is None else v * keep
    y = f["x"] + v * f["gate"][group] * f["scale"]
    u = _rms(y, f["w_next"])
    if not c["train"]:
        return y, u
    leaves = [f[k] for k in ("x", "h", "w", "gate", "scale", "w_next")]
    return (y.detach(), u.detach()) + torch.autograd.grad((y, u), leaves, (f["gy"], f["gu"]))
