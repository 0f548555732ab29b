"""What is measured of the operators of a worker's local step: the products grouped by worker, the
group norm with its activation, and the clipping of the workers' gradients.

Each case is one operator at one set of sizes.  `run` computes it in elementary torch operations, in 32
bits, or, where `own` is true, by the library's entry points.  Ragged counts (rows of a worker, tensors
of a vector) are a function of the case alone, values of the seed alone.
"""
import math
import random

import torch

own = False

DEV = "cuda"
F32, BF16 = "f32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}


def listed():
    return [
        # one sample for each of 16 workers through a square layer of a BERT-large sized model
        # (hidden width 1024): every worker's own weights are read for one row
        dict(name="linear_one_row", op="linear", dtype=BF16, out=BF16, workers=16, lo=1, hi=1, n_in=1024,
             n_out=1024, pad=0, mix=1),
        # the wide layer of the same model, forward, with the sample counts of workload 2
        dict(name="linear_wide", op="linear", dtype=BF16, out=BF16, workers=16, lo=500, hi=1500, n_in=1024,
             n_out=4096, pad=4096, mix=2),
        # gradient of the samples through a 2048 -> 1000 classifier, 32 workers with small batches
        dict(name="linear_dx_classifier", op="linear_dx", dtype=BF16, out=BF16, workers=32, lo=20, hi=300,
             n_in=2048, n_out=1000, pad=1000, mix=3),
        # gradient of the wide layer's weights, kept in 32 bits as the fused step takes it
        dict(name="linear_dw_wide", op="linear_dw", dtype=BF16, out=F32, workers=16, lo=500, hi=1500, n_in=4096,
             n_out=1024, pad=1024, mix=4),
        # forward of a 512 -> 1000 classifier in 32 bits, 32 workers
        dict(name="linear_f32", op="linear", dtype=F32, out=F32, workers=32, lo=500, hi=1500, n_in=512,
             n_out=1000, pad=1000, mix=5),
        # evaluation of one sample by each of 8 workers in the last block of a small residual network
        dict(name="norm_one_sample", op="norm", dtype=F32, params=F32, workers=8, lo=1, hi=1, length=49, channels=512,
             groups=32, act="relu", wider=0, mix=6),
        # training batches in the first block of a bottleneck network: 56 x 56 positions
        dict(name="norm_large_image", op="norm", dtype=BF16, params=F32, workers=8, lo=2, hi=8, length=3136,
             channels=256, groups=32, act="relu", wider=0, mix=7),
        # backward in the second stage of a small residual network, in 32 bits
        dict(name="norm_back_f32", op="norm_back", dtype=F32, params=F32, workers=16, lo=2, hi=12, length=784,
             channels=128, groups=32, act="silu", wider=0, mix=8),
        # backward in the third stage of a bottleneck network
        dict(name="norm_back_bf16", op="norm_back", dtype=BF16, params=F32, workers=16, lo=2, hi=12, length=196,
             channels=1024, groups=32, act="relu", wider=0, mix=9),
        # workload 1's vectors as gradients: 8 workers of 1 M numbers
        dict(name="clip_1m", op="clip", dtype=F32, workers=8, size=1_048_576, tensors=60, mix=10),
        # workload 2's vectors as gradients, in the 62 tensors of a ResNet-18
        dict(name="clip_resnet18", op="clip", dtype=F32, workers=32, size=11_689_512, tensors=62, mix=11),
        # workload 4's vectors (rows that are not 16-byte aligned) as gradients of 16 workers
        dict(name="clip_bf16", op="clip", dtype=BF16, workers=16, size=23_520_842, tensors=161, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: most are multiples of 8, some are odd."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.25 else max(8, v // 8 * 8)


def draw(rng):
    op = rng.choice(["linear", "linear_dx", "linear_dw", "norm", "norm_back", "clip"])
    mix = rng.randrange(1 << 20)
    if op.startswith("linear"):
        while True:
            dtype = rng.choice([BF16, BF16, BF16, F32])
            out = F32 if dtype == F32 or op == "linear_dw" and rng.random() < 0.5 else BF16
            hi = _log(rng, 1, 1500)
            case = dict(op=op, dtype=dtype, out=out, workers=_log(rng, 1, 64), lo=rng.randint(0, hi), hi=hi,
                        n_in=_width(rng, 24, 4096), n_out=_width(rng, 10, 4096), pad=_width(rng, 8, 4096), mix=mix)
            w = work(case)
            if sum(_counts(case)) > 0 and w["flops"] < (1.3e11 if dtype == BF16 else 3.2e10) and w["bytes"] < 6e8:
                return case
    if op.startswith("norm"):
        while True:
            groups = rng.choice([1, 2, 4, 8, 16, 32])
            hi = _log(rng, 1, 16)
            case = dict(op=op, dtype=rng.choice([F32, BF16]), params=rng.choice([F32, F32, BF16]),
                        workers=_log(rng, 1, 32), lo=rng.randint(0, hi), hi=hi,
                        length=_log(rng, 1, 3136), channels=groups * _log(rng, 1, 64), groups=groups,
                        act=rng.choice(["none", "relu", "silu"]), wider=rng.choice([0, 0, 8, 5]), mix=mix)
            if 0 < sum(_counts(case)) and 2 < case["length"] * case["channels"] // groups and work(case)["bytes"] < 1.5e8:
                return case
    while True:
        case = dict(op=op, dtype=rng.choice([F32, BF16]), workers=_log(rng, 1, 128), size=_log(rng, 1000, 24_000_000),
                    tensors=_log(rng, 1, 400), mix=mix)
        if work(case)["bytes"] < 2.9e9 and case["tensors"] * 4 < case["size"]:
            return case


def _counts(case):
    """Rows (or samples) of every worker."""
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["workers"])]


def _cuts(case):
    """Where the tensors of one vector begin, and its end."""
    r = random.Random(case["mix"])
    share = [math.exp(r.uniform(0, 7)) for _ in range(case["tensors"])]
    room, at, got = case["size"] - case["tensors"], 0.0, [0]
    for k, s in enumerate(share):
        at += s / sum(share)
        got.append(min(int(at * room) + k + 1, case["size"]))
    got[-1] = case["size"]
    return got


def work(case):
    if case["op"] == "clip":
        n = case["workers"] * case["size"]
        return {"bytes": 2.0 * n * SIZE[case["dtype"]] + 8 * case["workers"], "flops": 3.0 * n}
    counts = _counts(case)
    rows, e = sum(counts), SIZE[case["dtype"]]
    if case["op"].startswith("norm"):
        n = rows * case["length"] * case["channels"]
        par = case["workers"] * case["channels"] * 2 * SIZE[case["params"]]
        stats = rows * case["groups"] * 8
        if case["op"] == "norm":
            return {"bytes": 2.0 * n * e + par + stats, "flops": 8.0 * n}
        return {"bytes": 3.0 * n * e + par + stats + case["workers"] * case["channels"] * 8, "flops": 20.0 * n}
    k, n, o = case["n_in"], case["n_out"], SIZE[case["out"]]
    used = case["workers"] if case["op"] == "linear_dw" else sum(c > 0 for c in counts)
    sides = {"linear": rows * k * e + used * k * n * e + rows * n * o,
             "linear_dx": rows * n * e + used * k * n * e + rows * k * o,
             "linear_dw": rows * n * e + rows * k * e + used * k * n * o}
    return {"bytes": float(sides[case["op"]]), "flops": 2.0 * rows * k * n}


def _begins(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return torch.tensor(at, dtype=torch.int64, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype or t)

    if case["op"] == "clip":
        N, P = case["workers"], case["size"]
        # a gradient's size differs from worker to worker: some are clipped, some are not
        scale = torch.exp(torch.randn(N, 1, generator=g, device=DEV)) * 1e-3
        grads = torch.empty(N, P, dtype=t, device=DEV)
        torch.randn(N, P, generator=g, device=DEV, dtype=t, out=grads)
        grads.mul_(scale.to(t))
        out = torch.empty_like(grads)
        cuts = torch.tensor(_cuts(case), dtype=torch.int64)
        at = (torch.arange(N)[:, None] * P + cuts[None, :-1]).reshape(-1)
        begin = torch.cat([at, torch.tensor([N * P])]).to(DEV)
        rows = torch.arange(N + 1, dtype=torch.int32, device=DEV) * case["tensors"]
        e = grads.element_size()
        return dict(case=case, grads=grads, out=out, begin=begin, first=rows, max_norm=1e-3 * math.sqrt(P),
                    tensors=(grads.data_ptr() + at * e).to(DEV), outs=(out.data_ptr() + at * e).to(DEV),
                    norm=torch.empty(N, device=DEV), coef=torch.empty(N, device=DEV))
    counts = _counts(case)
    N, rows, begin = case["workers"], sum(counts), _begins(counts)
    if case["op"].startswith("norm"):
        L, C, G = case["length"], case["channels"], case["groups"]
        wide = C + case["wider"]
        p = TYPES[case["params"]]
        # what a convolution leaves: a mean of its own in every channel
        x = (torch.randn(rows, L, wide, generator=g, device=DEV) + torch.randn(wide, generator=g, device=DEV)).to(t)
        # gamma and beta lie in every worker's flat vector, other parameters between and behind them
        flat = torch.randn(N, 2 * C + 6, generator=g, device=DEV) * 0.2
        flat[:, :C] += 1.0
        flat = flat.to(p)
        s = dict(case=case, begin=begin, x=x[:, :, :C], gamma=flat[:, :C], beta=flat[:, C + 2:2 * C + 2],
                 y=torch.empty(rows, L, C, dtype=t, device=DEV), mean=torch.empty(rows, G, device=DEV),
                 rstd=torch.empty(rows, G, device=DEV))
        if case["op"] == "norm_back":
            s["dy"] = normal(rows, L, C)
            xs = s["x"].double().reshape(rows, L, G, C // G)
            var, mean = torch.var_mean(xs, dim=(1, 3), correction=0)
            s["mean"], s["rstd"] = mean.float(), torch.rsqrt(var + EPS).float()
            s["dgamma"], s["dbeta"] = torch.empty(N, C, device=DEV), torch.empty(N, C, device=DEV)
        return s
    k, n = case["n_in"], case["n_out"]
    s = dict(case=case, begin=begin, rows=rows, most=max(counts))
    o = TYPES[case["out"]]
    if case["op"] != "linear_dw":
        # the layer's weights lie in every worker's flat vector, other parameters behind them
        flat = normal(N, n * k + case["pad"], scale=1.0 / math.sqrt(k))
        s["w"] = flat[:, :n * k].unflatten(1, (n, k))
    if case["op"] != "linear_dx":
        s["x"] = normal(rows, k)
    if case["op"] != "linear":
        s["dy"] = normal(rows, n)
    if case["op"] == "linear_dw":
        s["out"] = torch.zeros(N, n * k + case["pad"], dtype=o, device=DEV)[:, :n * k].unflatten(1, (n, k))
    else:
        s["out"] = torch.empty(rows, n if case["op"] == "linear" else k, dtype=o, device=DEV)
    return s


EPS = 1e-5
ACT = {"none": 0, "relu": 1, "silu": 2}


def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state, op)
    if op == "clip":
        return _plain_clip(state)
    if op.startswith("norm"):
        return _plain_norm(state, op == "norm_back")
    return _plain_linear(state, op)


# ---------------------------------------------------------------- the library's entry points
def _own(s, op):
    import paper_1908_07782_b200 as combo

    c = s["case"]
    N = c["workers"]
    if op == "clip":
        if "scratch" not in s:
            s["scratch"] = torch.empty(combo.combo_grad_scratch_bytes(N), dtype=torch.uint8, device=DEV)
        combo.combo_grad_clip(s["tensors"], s["outs"], s["begin"], s["first"], len(s["tensors"]), N, N * c["size"],
                              s["grads"].element_size(), s["max_norm"], s["norm"], s["coef"], s["scratch"])
        return {"norm": s["norm"], "out": s["out"]}
    if op == "linear":
        combo.combo_grouped_linear(s["x"], s["w"], s["out"], s["begin"])
        return s["out"]
    if op == "linear_dx":
        combo.combo_grouped_linear_grad_input(s["dy"], s["w"], s["out"], s["begin"])
        return s["out"]
    if op == "linear_dw":
        combo.combo_grouped_linear_grad_weight(s["dy"], s["x"], s["out"], s["begin"])
        return s["out"]
    x = s["x"]
    if "scratch" not in s:
        need = combo.combo_group_norm_scratch_bytes(x.shape[0], x.shape[1], x.shape[2], c["groups"])
        s["scratch"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    if op == "norm":
        combo.combo_group_norm(x, s["y"], s["gamma"], s["beta"], s["begin"], c["groups"], EPS, ACT[c["act"]], s["mean"],
                               s["rstd"], s["scratch"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    combo.combo_group_norm_backward(s["dy"], x, s["y"], s["gamma"], s["beta"], s["begin"], c["groups"], ACT[c["act"]],
                                    s["mean"], s["rstd"], s["dgamma"], s["dbeta"], s["scratch"])
    return {"dx": s["y"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


# ---------------------------------------------------------------- plain forms
def _plain_clip(s):
    g = s["grads"].float()
    norm = (g * g).sum(1).sqrt()
    coef = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    return {"norm": norm, "out": (g * coef[:, None]).to(s["grads"].dtype)}


def _owners(begin, rows):
    """The worker that each row belongs to."""
    return torch.searchsorted(begin, torch.arange(rows, device=begin.device), right=True) - 1


def _plain_linear(s, op):
    begin, out = s["begin"], s["out"]
    # every worker's rows, side by side, as many as the worker with the most has
    at = begin[:-1, None] + torch.arange(s["most"], device=begin.device)
    mine = at < begin[1:, None]
    at = at.clamp(max=s["rows"] - 1)
    if op == "linear_dw":
        dy = s["dy"][at].float() * mine[:, :, None]
        return torch.bmm(dy.transpose(1, 2), s["x"][at].float()).to(out.dtype)
    w = s["w"].float()
    got = torch.bmm(s["x"][at].float(), w.transpose(1, 2)) if op == "linear" else torch.bmm(s["dy"][at].float(), w)
    who = _owners(begin, s["rows"])
    return got[who, torch.arange(s["rows"], device=begin.device) - begin[who]].to(out.dtype)


def _plain_norm(s, back):
    c, x = s["case"], s["x"].float()
    B, L, C = x.shape
    G = c["groups"]
    who = _owners(s["begin"], B)
    gamma, beta = s["gamma"].float()[who][:, None, :], s["beta"].float()[who][:, None, :]
    xg = x.reshape(B, L, G, C // G)
    if not back:
        mean = xg.mean(dim=(1, 3))
        d = xg - mean[:, None, :, None]
        rstd = torch.rsqrt((d * d).mean(dim=(1, 3)) + EPS)
        z = (d * rstd[:, None, :, None]).reshape(B, L, C) * gamma + beta
        y = z if c["act"] == "none" else z.clamp(min=0.0) if c["act"] == "relu" else z / (1.0 + torch.exp(-z))
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    mean, rstd = s["mean"][:, None, :, None], s["rstd"][:, None, :, None]
    xhat = ((xg - mean) * rstd).reshape(B, L, C)
    dz = s["dy"].float()
    if c["act"] != "none":
        z = xhat * gamma + beta
        if c["act"] == "relu":
            dz = dz * (z > 0)
        else:
            sig = 1.0 / (1.0 + torch.exp(-z))
            dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    dg = torch.zeros(c["workers"], C, device=DEV).index_add_(0, who, (dz * xhat).sum(1))
    db = torch.zeros(c["workers"], C, device=DEV).index_add_(0, who, dz.sum(1))
    t = (dz * gamma).reshape(B, L, G, C // G)
    h = xhat.reshape(B, L, G, C // G)
    m1 = t.mean(dim=(1, 3), keepdim=True)
    m2 = (t * h).mean(dim=(1, 3), keepdim=True)
    dx = (rstd * (t - m1 - h * m2)).reshape(B, L, C)
    return {"dx": dx.to(s["x"].dtype), "dgamma": dg, "dbeta": db}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        norms, outs = [], []
        for g in s["grads"]:
            g = g.double()
            norms.append(torch.linalg.vector_norm(g))
            outs.append(g * min(1.0, s["max_norm"] / (float(norms[-1]) + 1e-6)))
        return {"norm": torch.stack(norms), "out": torch.stack(outs)}
    at = s["begin"].tolist()
    spans = list(zip(at[:-1], at[1:]))
    if case["op"] == "linear":
        return torch.cat([s["x"][a:b].double() @ s["w"][w].double().T for w, (a, b) in enumerate(spans)])
    if case["op"] == "linear_dx":
        return torch.cat([s["dy"][a:b].double() @ s["w"][w].double() for w, (a, b) in enumerate(spans)])
    if case["op"] == "linear_dw":
        return torch.stack([s["dy"][a:b].double().T @ s["x"][a:b].double() for a, b in spans])
    C, G, act = case["channels"], case["groups"], case["act"]
    pieces = []
    for w, (a, b) in enumerate(spans):
        x = s["x"][a:b].double()
        h = x.unflatten(2, (G, C // G))
        var, mean = torch.var_mean(h, dim=(1, 3), correction=0, keepdim=True)
        rstd = 1.0 / torch.sqrt(var + EPS)
        if case["op"] == "norm_back":      # the statistics are inputs
            mean, rstd = (s[k][a:b].double()[:, None, :, None] for k in ("mean", "rstd"))
        h = ((h - mean) * rstd).flatten(2)
        z = h * s["gamma"][w].double() + s["beta"][w].double()
        sig = torch.sigmoid(z)
        if case["op"] == "norm":
            pieces.append((z if act == "none" else torch.relu(z) if act == "relu" else z * sig, mean.flatten(1), rstd.flatten(1)))
            continue
        slope = 1.0 if act == "none" else (z > 0).double() if act == "relu" else sig + z * sig * (1.0 - sig)
        dz = s["dy"][a:b].double() * slope
        t = (dz * s["gamma"][w].double()).unflatten(2, (G, C // G))
        hg = h.unflatten(2, (G, C // G))
        dx = rstd * (t - t.mean((1, 3), keepdim=True) - hg * (t * hg).mean((1, 3), keepdim=True))
        pieces.append((dx.flatten(2), (dz * h).sum((0, 1)), dz.sum((0, 1))))
    if case["op"] == "norm":
        y, mean, rstd = (torch.cat(v) for v in zip(*pieces))
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dg, db = zip(*pieces)
    return {"dx": torch.cat(dx), "dgamma": torch.stack(dg), "dbeta": torch.stack(db)}
