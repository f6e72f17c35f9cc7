"""Cases of use of the operators around experts, for timing and checking them.

Each case is one pass of a user's program through one operator: the layer norm,
rows sorted by expert and brought back with weights, and the experts' gated
feed-forward blocks on rows so sorted.  With `own` false a pass is the
operator's plain form: elementary torch operations in 32 bits, rounded once at
the end.  With `own` true it is the library's calls.

    listed()            the cases, dicts of plain values
    draw(rng)           one more case of the same ranges
    prepare(case, s)    inputs (and the plan) on the GPU, from the seed alone
    run(state)          one pass; returns its outputs
    work(case)          bytes and flops a pass cannot do without
    exact(case, s)      what run() returns, in 64 bits from the definitions
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5

# op "layer":    u = (x - mean) / sqrt(var + eps) * w + b of each row; train adds the gradients of x, w and b
# op "route":    the order of the rows by expert; x's rows in that order; rows in that order brought back, K a row, with
#                weights; train adds the gradient of the first and both of the second.  `none` is the share of the
#                choices that name no expert (beyond an expert's capacity, or a row that is switched off)
# op "experts":  Y = (act(X Wg^T) * (X Wu^T)) Wo^T by each expert's weights on the rows that chose it, in the sorted
#                order; train adds the gradients of X and of all weights


def listed():
    return [
        # one row normed: launch and latency
        {"name": "layer_serve_bf16_1x4096", "op": "layer", "train": False, "dtype": "bf16", "rows": 1, "width": 4096},
        # training, scalar features as wide as L = 16 rows
        {"name": "layer_train_fp32_8192x289", "op": "layer", "train": True, "dtype": "fp32", "rows": 8192,
         "width": 289},
        # training, ragged odd rows
        {"name": "layer_train_fp16_4001x1089", "op": "layer", "train": True, "dtype": "fp16", "rows": 4001,
         "width": 1089},
        # training, a long batch of wide rows
        {"name": "layer_train_bf16_16384x4096", "op": "layer", "train": True, "dtype": "bf16", "rows": 16384,
         "width": 4096},
        # one row to two of eight experts and back: launches and latency
        {"name": "route_serve_bf16_1x4096", "op": "route", "train": False, "dtype": "bf16", "rows": 1, "width": 4096,
         "per_row": 2, "experts": 8, "skew": 0.5, "none": 0.0},
        # training, odd sizes, some choices beyond their expert's capacity
        {"name": "route_train_fp32_4001x1089", "op": "route", "train": True, "dtype": "fp32", "rows": 4001,
         "width": 1089, "per_row": 3, "experts": 7, "skew": 1.0, "none": 0.1},
        # training, a long batch over many experts
        {"name": "route_train_bf16_16384x4096", "op": "route", "train": True, "dtype": "bf16", "rows": 16384,
         "width": 4096, "per_row": 2, "experts": 64, "skew": 0.5, "none": 0.0},
        # one row served by two of eight experts: their weights are all there is to read
        {"name": "experts_serve_bf16_1x2048x4096", "op": "experts", "train": False, "dtype": "bf16", "rows": 1,
         "d_in": 2048, "d_ff": 4096, "d_out": 2048, "act": "silu", "per_row": 2, "experts": 8, "skew": 0.5},
        # a small batch served together: a few rows an expert
        {"name": "experts_serve_bf16_64x2048x4096", "op": "experts", "train": False, "dtype": "bf16", "rows": 64,
         "d_in": 2048, "d_ff": 4096, "d_out": 2048, "act": "silu", "per_row": 2, "experts": 16, "skew": 0.5},
        # a ragged batch of L = 32 feature rows, every size odd or unaligned
        {"name": "experts_serve_fp16_1001x1089x725", "op": "experts", "train": False, "dtype": "fp16", "rows": 1001,
         "d_in": 1089, "d_ff": 725, "d_out": 1089, "act": "gelu", "per_row": 2, "experts": 6, "skew": 1.0},
        # training the blocks that make the path weights of 8192 pairs at L = 16, a block for each kind of pair
        {"name": "experts_train_fp32_8192x128x512x3281", "op": "experts", "train": True, "dtype": "fp32",
         "rows": 8192, "d_in": 128, "d_ff": 512, "d_out": 3281, "act": "silu", "per_row": 1, "experts": 5,
         "skew": 1.0},
        # a training step of large blocks: the most arithmetic
        {"name": "experts_train_bf16_8192x2048x4096", "op": "experts", "train": True, "dtype": "bf16", "rows": 8192,
         "d_in": 2048, "d_ff": 4096, "d_out": 2048, "act": "silu", "per_row": 2, "experts": 16, "skew": 0.5},
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; half of the larger ones are multiples of 8."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = max(lo, min(hi, n))
    return n // 8 * 8 if n >= 64 and rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["layer", "route", "experts", "experts"])
    c = {"op": op, "train": rng.random() < 0.6, "dtype": rng.choice(["fp32", "bf16", "fp16"])}
    if op == "layer":
        c["width"] = _log(rng, 16, 16384)
        c["rows"] = max(1, min(_log(rng, 1, 65536), 16384 * 4096 // c["width"]))
        return c
    c["experts"] = _log(rng, 2, 64) if op == "experts" else _log(rng, 2, 256)
    c["per_row"] = rng.randint(1, min(4, c["experts"])) if op == "experts" else rng.randint(1, min(8, c["experts"]))
    c["skew"] = rng.choice([0.0, 0.5, 1.0])
    if op == "route":
        c["width"] = _log(rng, 16, 8192)
        c["rows"] = max(1, min(_log(rng, 1, 65536), 16384 * 4096 * 2 // (c["width"] * c["per_row"])))
        c["none"] = rng.choice([0.0, 0.0, 0.1, 0.5])
        return c
    c["d_in"], c["d_ff"] = _log(rng, 64, 2048), _log(rng, 64, 4096)
    c["d_out"] = c["d_in"] if rng.random() < 0.5 else _log(rng, 64, 2048)
    sizes = c["d_ff"] * (2 * c["d_in"] + c["d_out"])
    # within the largest listed case; 32-bit blocks are those of path weights, a thirtieth of its work
    c["experts"] = max(2, min(c["experts"], 16 * 4096 * 3 * 2048 // sizes))
    c["per_row"] = min(c["per_row"], c["experts"])
    most = 2.4e12 if c["dtype"] != "fp32" else 8e10
    c["rows"] = max(1, min(_log(rng, 1, 8192), int(most / (6 * sizes * c["per_row"]))))
    c["act"] = rng.choice(["silu", "gelu", "relu"])
    return c


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale + mean).to(dt)

    s, n = {"case": case}, case["rows"]
    if case["op"] == "layer":
        d = case["width"]
        s["x"] = normal(n, d, mean=0.5)
        s["w"], s["b"] = normal(d, scale=0.1, mean=1.0), normal(d, scale=0.1)
        if case["train"]:
            s["gu"] = normal(n, d)
        if own:
            import paper_2602_21466_amd as lib
            s["plan"] = lib.LayerNormPlan(d, dtype=case["dtype"], eps=EPS)
        return s
    k, experts = case["per_row"], case["experts"]
    # a router's choice: the k largest of each row's scores, some experts chosen more often than others
    scores = torch.randn(n, experts, generator=g, device=dev)
    scores = scores + case["skew"] * torch.randn(experts, generator=g, device=dev)
    top, s["index"] = torch.topk(scores, k, dim=1)
    s["weights"] = torch.softmax(top, 1)
    if case["op"] == "route":
        d = case["width"]
        if case["none"] > 0:
            s["index"] = torch.where(torch.rand(n, k, generator=g, device=dev) < case["none"], -1, s["index"])
        s["x"], s["ys"] = normal(n, d), normal(n * k, d)
        if case["train"]:
            s["gxs"], s["gy"] = normal(n * k, d), normal(n, d)
        return s
    di, df, do = case["d_in"], case["d_ff"], case["d_out"]
    s["x"] = normal(n, di)  # features as a norm leaves them
    s["w_in"] = normal(experts, 2 * df, di, scale=di ** -0.5)
    s["w_out"] = normal(experts, do, df, scale=df ** -0.5)
    if case["train"]:
        s["gy"] = normal(n * k, do)
    # the order of the rows, made before: it is the other operator's work
    if own:
        import paper_2602_21466_amd as lib
        s["routes"] = lib.Routes(s["index"], experts)
        s["plan"] = lib.ExpertsPlan(experts, di, df, do, dtype=case["dtype"], activation=case["act"])
    else:
        flat = s["index"].flatten()
        s["order"] = torch.argsort(flat, stable=True)
        s["counts"] = torch.bincount(flat, minlength=experts).tolist()
    return s


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2602_21466_amd as lib
    c, train = s["case"], s["case"]["train"]
    if c["op"] == "layer":
        u, stats = s["plan"].forward(s["x"], s["w"], s["b"])
        return (u,) + tuple(s["plan"].backward(s["x"], s["w"], stats, s["gu"])) if train else u
    if c["op"] == "route":
        r = lib.Routes(s["index"], c["experts"])
        out = (r.place, r.source, r.offsets, r.gather(s["x"]), r.combine(s["ys"], s["weights"]))
        if not train:
            return out
        return out + (r.gather_backward(s["gxs"]),) + tuple(r.combine_backward(s["ys"], s["weights"], s["gy"]))
    if not train:
        return s["plan"].forward(s["x"], s["routes"], s["w_in"], s["w_out"])
    y, saved = s["plan"].forward(s["x"], s["routes"], s["w_in"], s["w_out"], save=True)
    return (y,) + tuple(s["plan"].backward(s["x"], s["routes"], s["w_in"], s["w_out"], saved, s["gy"]))


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


def _run_plain(s):
    c, train = s["case"], s["case"]["train"]
    dt = DTYPES[c["dtype"]]
    f = {k: v.float() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if c["op"] == "layer":
        x, w = f["x"], f["w"]
        x = x - x.mean(1, keepdim=True)
        r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
        v = x * r
        u = (v * w + f["b"]).to(dt)
        if not train:
            return u
        a = f["gu"] * w
        gx = r * (a - a.mean(1, keepdim=True) - v * (a * v).mean(1, keepdim=True))
        return u, gx.to(dt), (f["gu"] * v).sum(0).to(dt), f["gu"].sum(0).to(dt)
    if c["op"] == "route":
        n, k, experts = c["rows"], c["per_row"], c["experts"]
        index = s["index"]
        valid = index >= 0
        key = torch.where(valid, index, experts).flatten()
        order = torch.argsort(key, stable=True)
        at = torch.arange(n * k, device=key.device)
        offsets = (key[:, None] < torch.arange(experts + 1, device=key.device)).sum(0)
        held = at < offsets[experts]
        source = torch.where(held, order, -1)
        place = torch.empty_like(order)
        place[order] = at
        place = torch.where(valid, place.reshape(n, k), -1)
        xs = torch.where(held[:, None], s["x"][order // k], 0.0)
        w, mask, from_ = f["weights"][:, :, None], valid[:, :, None], place.clamp_min(0)
        rows = torch.where(mask, f["ys"][from_], 0.0)
        y = (w * rows).sum(1).to(dt)
        out = place.int(), source.int(), offsets.int(), xs, y
        if not train:
            return out
        gx = torch.where(mask, f["gxs"][from_], 0.0).sum(1).to(dt)
        gw = (rows * f["gy"][:, None, :]).sum(2)
        gys = torch.where(held[:, None], f["weights"].flatten()[order][:, None] * f["gy"][order // k], 0.0).to(dt)
        return out + (gx, gys, gw)
    k, df = c["per_row"], c["d_ff"]
    token = s["order"] // k
    xs, ys, first = f["x"][token], [], 0
    gxs, gw_in, gw_out = [], [], []
    for e, count in enumerate(s["counts"]):
        x, w_in, w_out = xs[first:first + count], f["w_in"][e], f["w_out"][e]
        gate, up = x @ w_in[:df].T, x @ w_in[df:].T
        a, da = _act(gate, c["act"])
        h = a * up
        ys.append(h @ w_out.T)
        if train:
            gy = f["gy"][first:first + count]
            dh = gy @ w_out
            d = torch.cat([dh * up * da, dh * a], 1)
            gxs.append(d @ w_in)
            gw_in.append(d.T @ x)
            gw_out.append(gy.T @ h)
        first += count
    y = torch.cat(ys).to(dt)
    if not train:
        return y
    gx = torch.zeros_like(f["x"]).index_add_(0, token, torch.cat(gxs))
    return y, gx.to(dt), torch.stack(gw_in).to(dt), torch.stack(gw_out).to(dt)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    e, n = SIZE[case["dtype"]], case["rows"]
    if case["op"] == "layer":
        d = case["width"]
        # x in, u out; gradients: gu in, gx out (x is read once in all), weight and bias and their gradients
        return {"flops": n * d * (18.0 if case["train"] else 7.0),
                "bytes": e * ((4 * n + 4) * d if case["train"] else (2 * n + 2) * d)}
    k, experts = case["per_row"], case["experts"]
    held = n * k * (1.0 - case.get("none", 0.0))  # choices that name an expert
    if case["op"] == "route":
        d, order = case["width"], (8 + 4 + 4 + 4) * n * k  # the choices (64 bits), place, source, weights
        if not case["train"]:
            # x in, its rows out (all n k are written); the experts' rows in, y out
            return {"flops": 2.0 * held * d, "bytes": e * d * (2 * n + n * k + held) + order}
        # and their gradients' rows in, gx out; gy in, the rows' gradients out, and the weights'
        return {"flops": 6.0 * held * d, "bytes": e * d * (4 * n + 2 * n * k + 2 * held) + order + 4 * n * k}
    di, df, do = case["d_in"], case["d_ff"], case["d_out"]
    flops = 2.0 * n * k * df * (2 * di + do)
    # experts with a row, were all chosen alike
    chosen = experts * (1.0 - (1.0 - k / experts) ** n)
    if case["train"]:
        # forward, and twice its products backward; x, y, gy, gx once each, weights, and every expert's gradients
        return {"flops": 3 * flops,
                "bytes": e * (2 * n * di + 2 * n * k * do + (chosen + experts) * df * (2 * di + do))}
    return {"flops": flops, "bytes": e * (n * di + n * k * do + chosen * df * (2 * di + do))}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    f = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if c["op"] == "layer":
        leaves = [f[k].requires_grad_(c["train"]) for k in ("x", "w", "b")]
        var, mean = torch.var_mean(leaves[0], 1, correction=0, keepdim=True)
        u = (leaves[0] - mean) / (var + EPS).sqrt() * leaves[1] + leaves[2]
        return (u.detach(),) + torch.autograd.grad(u, leaves, f["gu"]) if c["train"] else u
    n, k, experts = c["rows"], c["per_row"], c["experts"]
    index = s["index"].cpu().numpy().reshape(-1)
    lists = [(index == e).nonzero()[0].tolist() for e in range(experts)]
    source = [slot for rows in lists for slot in rows]
    bounds = [0]
    for rows in lists:
        bounds.append(bounds[-1] + len(rows))
    order = torch.tensor(source, dtype=torch.int64, device="cuda")
    if c["op"] == "route":
        place = torch.full((n * k,), -1, dtype=torch.int32, device="cuda")
        place[order] = torch.arange(len(source), dtype=torch.int32, device="cuda")
        out_source = torch.full((n * k,), -1, dtype=torch.int32, device="cuda")
        out_source[:len(source)] = order.int()
        xs = torch.zeros(n * k, c["width"], dtype=torch.float64, device="cuda")
        xs[:len(source)] = f["x"][order // k]
        wsort = f["weights"].reshape(-1)[order]
        ys = f["ys"][:len(source)]
        y = torch.zeros_like(f["x"]).index_add_(0, order // k, wsort[:, None] * ys)
        out = place.reshape(n, k), out_source, torch.tensor(bounds, dtype=torch.int32, device="cuda"), xs, y
        if not c["train"]:
            return out
        gx = torch.zeros_like(f["x"]).index_add_(0, order // k, f["gxs"][:len(source)])
        gys = torch.zeros_like(f["ys"])
        gy = f["gy"][order // k]
        gys[:len(source)] = wsort[:, None] * gy
        gw = torch.zeros(n * k, dtype=torch.float64, device="cuda")
        gw[order] = torch.linalg.vecdot(gy, ys)
        return out + (gx, gys, gw.reshape(n, k))
    act = {"silu": lambda v: v * torch.sigmoid(v), "relu": lambda v: v.clamp_min(0.0),
           "gelu": lambda v: v * torch.special.ndtr(v)}[c["act"]]
    y = torch.empty(n * k, c["d_out"], dtype=torch.float64, device="cuda")
    gx, gwi, gwo = torch.zeros_like(f["x"]), torch.zeros_like(f["w_in"]), torch.zeros_like(f["w_out"])
    for e in range(experts):
        at = slice(bounds[e], bounds[e + 1])
        token = order[at] // k
        leaves = [t.requires_grad_(c["train"]) for t in (f["x"][token], f["w_in"][e].clone(), f["w_out"][e].clone())]
        a, b = (leaves[0] @ leaves[1].T).chunk(2, 1)
        ye = (act(a) * b) @ leaves[2].T
        y[at] = ye.detach()
        if c["train"]:
            ge = torch.autograd.grad(ye, leaves, f["gy"][at])
            gx.index_add_(0, token, ge[0])
            gwi[e], gwo[e] = ge[1], ge[2]
    return (y, gx, gwi, gwo) if c["train"] else y
