"""What is measured of the operators at the end and inside of a worker's local step: the softmax cross entropy of a
linear classifier over many classes, grouped by worker, without its logits being kept, forward and with its gradients;
and dropout whose mask comes from a counter-based generator and is never stored.

Each case is one operator at one set of sizes.  `run` computes it in elementary torch operations, in 32 bits, or, where
`own` is true, by the library's entry points.  Ragged counts and which rows have a label are a function of the case
alone, values (labels among them) of the seed alone.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
F32, BF16 = "f32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}


def listed():
    return [
        # the classifier of the local-training example, one sample a worker (an online step): all latency
        dict(name="loss_small_classifier", op="loss", dtype=F32, workers=8, lo=1, hi=1, n_in=256, classes=10, labelled=1.0,
             wide=0, pad=0, mix=1),
        # evaluation through a 512 -> 1000 classifier in 32 bits, sample counts of workload 2
        dict(name="loss_classifier_f32", op="loss", dtype=F32, workers=32, lo=500, hi=1500, n_in=512, classes=1000,
             labelled=1.0, wide=0, pad=1000, mix=2),
        # next-word loss of one token a worker at a BERT-large sized model's width: a pass over every worker's weights
        dict(name="loss_vocabulary_one_row", op="loss", dtype=BF16, workers=16, lo=1, hi=1, n_in=1024, classes=32000,
             labelled=1.0, wide=0, pad=1024, mix=3),
        # the same with a local step's tokens; a vocabulary that no tile divides
        dict(name="loss_vocabulary", op="loss", dtype=BF16, workers=8, lo=500, hi=1500, n_in=1024, classes=30001,
             labelled=1.0, wide=0, pad=1024, mix=4),
        # gradients of the example's classifier with its sample counts
        dict(name="back_small_classifier", op="back", dtype=F32, out=F32, workers=8, lo=100, hi=249, n_in=256, classes=10,
             labelled=1.0, grad="mean", wide=0, pad=0, mix=5),
        # gradients in 32 bits through a classifier over many classes
        dict(name="back_classes_f32", op="back", dtype=F32, out=F32, workers=8, lo=100, hi=500, n_in=512, classes=10000,
             labelled=1.0, grad="mean", wide=0, pad=512, mix=6),
        # masked words: 15 of 100 tokens carry a label, the others enter neither loss nor gradient
        dict(name="back_masked_words", op="back", dtype=BF16, out=BF16, workers=8, lo=1024, hi=4096, n_in=1024, classes=30001,
             labelled=0.15, grad="mean", wide=0, pad=1024, mix=7),
        # every token labelled; the weights' gradient in 32 bits, as clipping and the fused step take it
        dict(name="back_vocabulary", op="back", dtype=BF16, out=F32, workers=4, lo=1500, hi=2500, n_in=768, classes=32000,
             labelled=1.0, grad="rows", wide=8, pad=768, mix=8),
        # one sample a worker, the example's width
        dict(name="dropout_one_sample", op="dropout", dtype=F32, workers=8, lo=1, hi=1, width=256, p=0.1, residual=False,
             wide=0, mix=9),
        # activations of the wide layer of a BERT-large sized model, sample counts of workload 2
        dict(name="dropout_wide", op="dropout", dtype=BF16, workers=16, lo=500, hi=1500, width=4096, p=0.1, residual=False,
             wide=0, mix=10),
        # the end of a block: dropout of the branch, added to what came in
        dict(name="dropout_residual", op="dropout", dtype=BF16, workers=16, lo=1000, hi=3000, width=1024, p=0.1, residual=True,
             wide=0, mix=11),
        # activations of a convolution's 28 x 28 positions in 32 bits
        dict(name="dropout_f32", op="dropout", dtype=F32, workers=16, lo=1568, hi=9408, width=128, p=0.25, residual=False,
             wide=0, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: most are multiples of 8, some are odd."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.25 else max(8, v // 8 * 8)


def draw(rng):
    op = rng.choice(["loss", "back", "back", "dropout"])
    mix = rng.randrange(1 << 20)
    if op == "dropout":
        while True:
            hi = _log(rng, 1, 10000)
            case = dict(op=op, dtype=rng.choice([F32, BF16]), workers=_log(rng, 1, 64), lo=rng.randint(0, hi), hi=hi,
                        width=_width(rng, 10, 4096), p=rng.choice([0.0, 0.05, 0.1, 0.25, 0.5]), residual=rng.random() < 0.5,
                        wide=rng.choice([0, 0, 8, 5]), mix=mix)
            if sum(_counts(case)) > 0 and work(case)["bytes"] < 2.6e8:
                return case
    while True:
        hi = _log(rng, 1, 4096)
        dtype = rng.choice([F32, BF16, BF16])
        case = dict(op=op, dtype=dtype, workers=_log(rng, 1, 64), lo=rng.randint(0, hi), hi=hi, n_in=_width(rng, 16, 2048),
                    classes=_log(rng, 4, 65536), labelled=rng.choice([1.0, 1.0, 0.5, 0.15]), wide=rng.choice([0, 0, 8, 5]),
                    pad=_width(rng, 8, 4096), mix=mix)
        if op == "back":
            case.update(out=F32 if dtype == F32 else rng.choice([F32, BF16]), grad=rng.choice(["mean", "rows"]))
        cost, rows = 2.0 * sum(_counts(case)) * case["n_in"] * case["classes"], sum(_labelled(case))
        limit = 4.5e11 if dtype == BF16 else 4e10
        if rows > 0 and cost < (limit if op == "loss" else limit / 1.2) and \
                work(case)["bytes"] < 1.04e9 and case["workers"] * hi * case["classes"] < 4e8:
            return case


def _counts(case):
    """Rows (samples, tokens) of every worker."""
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["workers"])]


def _labelled(case):
    """Whether a row has a label."""
    if case["labelled"] == 1.0:
        return np.ones(sum(_counts(case)), dtype=bool)
    return np.random.default_rng(case["mix"]).random(sum(_counts(case))) < case["labelled"]


def work(case):
    counts, e = _counts(case), SIZE[case["dtype"]]
    rows = sum(counts)
    if case["op"] == "dropout":
        n = rows * case["width"]
        return {"bytes": (2.0 + case["residual"]) * n * e, "flops": 2.0 * n}
    has = _labelled(case)
    some = int(has.sum())
    ends = np.cumsum(counts)
    used = sum(bool(has[b - c:b].any()) for b, c in zip(ends, counts))
    k, v = case["n_in"], case["classes"]
    if case["op"] == "loss":
        return {"bytes": float(some * k * e + used * k * v * e + rows * 16), "flops": 2.0 * some * k * v}
    return {"bytes": float((some + rows) * k * e + used * k * v * e + case["workers"] * k * v * SIZE[case["out"]] + rows * 16),
            "flops": 6.0 * some * k * v}


def _begins(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64), device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    counts = _counts(case)
    N, M, begin = case["workers"], sum(counts), _begins(counts)
    if case["op"] == "dropout":
        n = case["width"]

        def rows():
            return torch.randn(M, n + case["wide"], generator=g, device=DEV).to(t)[:, :n]

        return dict(case=case, counts=counts, begin=begin, x=rows(), residual=rows() if case["residual"] else None,
                    y=torch.empty(M, n, dtype=t, device=DEV), seed=random.Random(seed).getrandbits(64),
                    round=random.Random(seed + 1).getrandbits(32), site=random.Random(seed + 2).randrange(64))
    k, v = case["n_in"], case["classes"]
    s = dict(case=case, begin=begin, rows=M, most=max(counts))
    # a norm's output in front of the classifier
    s["x"] = torch.randn(M, k + case["wide"], generator=g, device=DEV).to(t)[:, :k]
    # the classifier's weights lie in every worker's flat vector, other parameters behind them; logits spread by 1.5
    flat = (torch.randn(N, v * k + case["pad"], generator=g, device=DEV) * (1.5 / math.sqrt(k))).to(t)
    s["w"] = flat[:, :v * k].unflatten(1, (v, k))
    # few of many classes are frequent
    u = torch.rand(M, generator=g, device=DEV, dtype=torch.float64)
    s["labels"] = (torch.exp(u * math.log(v + 1.0)) - 1.0).to(torch.int64).clamp_(0, v - 1)
    s["labels"][~torch.from_numpy(_labelled(case)).to(DEV)] = -100
    if case["op"] == "loss":
        s["loss"], s["lse"] = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        return s
    s["lse"] = torch.zeros(M, device=DEV)
    at = begin.tolist()
    for w, (a, b) in enumerate(zip(at[:-1], at[1:])):
        for c in range(a, b, 1024):
            s["lse"][c:min(c + 1024, b)] = torch.logsumexp(s["x"][c:min(c + 1024, b)].double() @ s["w"][w].double().T, 1).float()
    s["lse"][s["labels"] < 0] = 0.0
    s["row_grad"] = None if case["grad"] == "mean" else torch.rand(M, generator=g, device=DEV) / max(counts)
    s["dx"] = torch.empty(M, k, dtype=t, device=DEV)
    s["dw"] = torch.empty(N, v * k + case["pad"], dtype=TYPES[case["out"]], device=DEV)[:, :v * k].unflatten(1, (v, k))
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state, op)
    if op == "dropout":
        return _plain_dropout(state)
    return _plain_loss(state, op == "back")


# ---------------------------------------------------------------- the library's entry points
def _own(s, op):
    import paper_1908_07782_b200 as combo

    c = s["case"]
    if op == "dropout":
        combo.combo_dropout(s["x"], s["residual"], s["y"], s["begin"], c["p"], s["seed"], s["round"], s["site"])
        return s["y"]
    if "scratch" not in s:
        need = combo.combo_grouped_cross_entropy_scratch_bytes(c["workers"], s["rows"], c["n_in"], c["classes"], SIZE[c["dtype"]],
                                                               SIZE[c["out"]] if op == "back" else 0)
        s["scratch"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    if op == "loss":
        combo.combo_grouped_cross_entropy(s["x"], s["w"], s["labels"], s["loss"], s["lse"], s["begin"], s["scratch"])
        return {"loss": s["loss"], "lse": s["lse"]}
    combo.combo_grouped_cross_entropy_backward(s["x"], s["w"], s["labels"], s["lse"], s["row_grad"], s["dx"], s["dw"], s["begin"],
                                               s["scratch"])
    return {"dx": s["dx"], "dw": s["dw"]}


# ---------------------------------------------------------------- plain forms
def _owners(begin, rows):
    """The worker that each row belongs to."""
    return torch.searchsorted(begin, torch.arange(rows, device=begin.device), right=True) - 1


def _plain_loss(s, back):
    begin = s["begin"]
    # every worker's rows, side by side, as many as the worker with the most has
    at = begin[:-1, None] + torch.arange(s["most"], device=begin.device)
    mine = at < begin[1:, None]
    at = at.clamp(max=s["rows"] - 1)
    labels = s["labels"][at]
    has = mine & (labels >= 0)
    labels = labels.clamp(min=0)
    x = s["x"][at].float() * has[:, :, None]
    w = s["w"].float()
    z = torch.bmm(x, w.transpose(1, 2))
    who = _owners(begin, s["rows"])
    place = torch.arange(s["rows"], device=begin.device) - begin[who]
    if not back:
        most = z.max(2, keepdim=True).values
        lse = most[:, :, 0] + torch.log(torch.exp(z - most).sum(2))
        loss = lse - torch.gather(z, 2, labels[:, :, None])[:, :, 0]
        return {"loss": (loss * has)[who, place], "lse": (lse * has)[who, place]}
    if s["row_grad"] is None:
        scale = has.float() / has.sum(1, keepdim=True).clamp(min=1)
    else:
        scale = s["row_grad"][at] * has
    d = torch.exp(z.sub_(s["lse"][at][:, :, None]))
    d.scatter_add_(2, labels[:, :, None], torch.full_like(labels, -1.0, dtype=torch.float32)[:, :, None])
    d *= scale[:, :, None]
    dx = torch.bmm(d, w)[who, place]
    dw = torch.bmm(d.transpose(1, 2), x)
    return {"dx": dx.to(s["dx"].dtype), "dw": dw.to(s["dw"].dtype)}


MASK64 = (1 << 64) - 1
C0, C1, C2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _signed(v):
    v &= MASK64
    return v - (1 << 64) if v >> 63 else v


def _step(z):
    """One step of the splitmix64 generator from the state z: an int64 tensor, or a number."""
    if isinstance(z, int):
        z = (z + C0) & MASK64
        z = ((z ^ z >> 30) * C1) & MASK64
        z = ((z ^ z >> 27) * C2) & MASK64
        return z ^ z >> 31
    z = z + _signed(C0)
    z = (z ^ (z >> 30 & (1 << 34) - 1)) * _signed(C1)
    z = (z ^ (z >> 27 & (1 << 37) - 1)) * _signed(C2)
    return z ^ (z >> 31 & (1 << 33) - 1)


def _plain_dropout(s):
    c, x = s["case"], s["x"]
    M, n = x.shape
    lots = (n + 3) // 4                                 # a draw of 64 bits serves four neighbours of a row
    first = _step(s["seed"])
    keys = [_step(_step(first ^ (s["round"] << 32 | w)) ^ (0x80000000 << 32 | s["site"])) for w in range(c["workers"])]
    who = _owners(s["begin"], M)
    keys = torch.tensor([_signed(k) for k in keys], device=DEV)[who]
    row = torch.arange(M, device=DEV) - s["begin"][who]
    h = _step(keys[:, None] ^ (row[:, None] * lots + torch.arange(lots, device=DEV)))
    bits = torch.stack([h >> 16 * j & 0xffff for j in range(4)], 2).reshape(M, lots * 4)[:, :n]
    drop = int(c["p"] * 65536 + 0.5)
    y = torch.where(bits >= drop, x.float() * (65536.0 / (65536 - drop)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        return _exact_dropout(s)
    at = s["begin"].tolist()
    pieces, dws = [], []
    for w, (a, b) in enumerate(zip(at[:-1], at[1:])):
        weights = s["w"][w].double()
        dw = torch.zeros_like(weights)
        valued = max(int((s["labels"][a:b] >= 0).sum()), 1)
        for c0 in range(a, b, 1024):
            c1 = min(c0 + 1024, b)
            x, labels = s["x"][c0:c1].double(), s["labels"][c0:c1]
            has = labels >= 0
            logits = x @ weights.T
            if case["op"] == "loss":
                lse = torch.logsumexp(logits, 1)
                mine = logits[torch.arange(c1 - c0, device=DEV), labels.clamp(min=0)]
                pieces.append((torch.where(has, lse - mine, 0.0), torch.where(has, lse, 0.0)))
                continue
            soft = torch.exp(logits - s["lse"][c0:c1].double()[:, None])
            soft[torch.arange(c1 - c0, device=DEV), labels.clamp(min=0)] -= 1.0
            size = torch.full((c1 - c0,), 1.0 / valued, dtype=torch.float64, device=DEV) if s["row_grad"] is None else \
                s["row_grad"][c0:c1].double()
            soft *= torch.where(has, size, 0.0)[:, None]
            pieces.append(soft @ weights)
            dw += soft.T @ x
        dws.append(dw)
    if case["op"] == "loss":
        loss, lse = zip(*pieces)
        return {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return {"dx": torch.cat(pieces), "dw": torch.stack(dws)}


def _exact_dropout(s):
    c = s["case"]
    M, n = s["x"].shape
    u = np.uint64

    def mixed(z):
        with np.errstate(over="ignore"):
            z = z + u(C0)
            z = (z ^ (z >> u(30))) * u(C1)
            z = (z ^ (z >> u(27))) * u(C2)
            return z ^ (z >> u(31))

    lots, drop = -(-n // 4), int(c["p"] * 65536 + 0.5)
    keep = np.empty((M, n), dtype=bool)
    a = 0
    for w, count in enumerate(s["counts"]):
        key = mixed(mixed(np.array([s["seed"]], dtype=u)) ^ u(s["round"] << 32 | w))
        key = mixed(key ^ u(0x80000000 << 32 | s["site"]))
        drawn = mixed(np.arange(count * lots, dtype=u) ^ key).astype("<u8").view("<u2")
        keep[a:a + count] = drawn.reshape(count, lots * 4)[:, :n] >= drop
        a += count
    y = s["x"].double() * torch.from_numpy(keep).to(DEV) / (1.0 - drop / 65536.0)
    return y if s["residual"] is None else y + s["residual"].double()
