"""combo_dropout: its mask against the generator's definition, its arithmetic, and what it must not depend on."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
M64 = (1 << 64) - 1


def step(z):
    """splitmix64 from state z, numbers of any length."""
    z = (z + 0x9E3779B97F4A7C15) & M64
    z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ z >> 27) * 0x94D049BB133111EB) & M64
    return z ^ z >> 31


def kept(rows, n, p, seed, rnd, site, worker):
    T = int(p * 65536 + 0.5)
    key = step(step(step(seed) ^ (rnd << 32 | worker)) ^ (1 << 63 | site))
    lots = -(-n // 4)
    out = np.zeros((rows, n), dtype=bool)
    for r in range(rows):
        for lot in range(lots):
            h = step(key ^ (r * lots + lot))
            for c in range(4 * lot, min(4 * lot + 4, n)):
                out[r, c] = (h >> 16 * (c % 4)) % 65536 >= T
    return out


def array(M, n, pitch, dtype, skew, g):
    buf = torch.full((skew + M * pitch + 16,), float("nan"), dtype=dtype, device=DEV)
    t = buf[skew:skew + M * pitch].view(M, pitch)[:, :n]
    t.copy_(torch.randn(M, n, generator=g))
    return buf, t


SHAPES = {
    "one": dict(counts=[1], n=1), "narrow": dict(counts=[3, 0, 5], n=3), "vector": dict(counts=[2, 2], n=8),
    "odd": dict(counts=[4, 0, 0, 9, 1], n=37), "pitch": dict(counts=[6, 3], n=40, extra=8), "off 16 bytes": dict(counts=[6, 3], n=40, extra=3, skew=1),
    "row in pieces": dict(counts=[2, 1], n=2500), "odd in pieces": dict(counts=[1, 2], n=2501), "rows of none": dict(counts=[4, 4], n=24, lead=2, behind=3),
}


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_mask_and_values(shape, dtype, residual):
    counts, n, extra, skew, lead, behind = (SHAPES[shape].get(k, d) for k, d in
                                            (("counts", 0), ("n", 0), ("extra", 0), ("skew", 0), ("lead", 0), ("behind", 0)))
    p, seed, rnd, site = 0.3, (1 << 63) + 12345, 0xfffffff0, 7
    g = torch.Generator().manual_seed(n)
    M = lead + sum(counts) + behind
    _, x = array(M, n, n + extra, dtype, skew, g)
    r = array(M, n, n + extra, dtype, skew, g)[1] if residual else None
    buf, y = array(M, n, n + extra, dtype, skew, g)
    before = y.clone()
    at = lead + np.concatenate([[0], np.cumsum(counts)])
    mask = np.concatenate([kept(c, n, p, seed, rnd, site, w) for w, c in enumerate(counts)])
    keep = torch.from_numpy(mask).to(DEV)
    inside = slice(int(at[0]), int(at[-1]))
    # what is dropped may hold anything
    x[inside][~keep] = torch.tensor([float("nan"), float("inf")])[torch.arange(int((~keep).sum())) % 2].to(x)
    combo.combo_dropout(x, r, y, torch.tensor(at).to(DEV), p, seed, rnd, site)
    T = int(p * 65536 + 0.5)
    want = torch.where(keep, x[inside].float() * np.float32(65536 / (65536 - T)), 0.0)
    if residual:
        want = want + r[inside].float()
    assert torch.equal(y[inside], want.to(dtype))
    assert torch.equal(y[:lead], before[:lead]) and torch.equal(y[M - behind:], before[M - behind:])
    assert int((~buf.isnan()).sum()) == y.numel()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_workers_mask_is_its_own(dtype):
    """The same alone, among others, and numbered by first_worker; in place; backward the same mask."""
    counts, n = [5, 70, 0, 33], 136
    at = np.concatenate([[0], np.cumsum(counts)])
    x = torch.randn(sum(counts), n, device=DEV).to(dtype)
    y = torch.empty_like(x)
    combo.combo_dropout(x, None, y, torch.tensor(at).to(DEV), 0.2, 5, 6, 1)
    for w, c in enumerate(counts):
        part = x[at[w]:at[w + 1]].clone()
        combo.combo_dropout(part, None, part, None, 0.2, 5, 6, 1, first_worker=w)
        assert torch.equal(part, y[at[w]:at[w + 1]])
    dy = torch.randn_like(x)
    dx = torch.empty_like(x)
    combo.combo_dropout(dy, None, dx, torch.tensor(at).to(DEV), 0.2, 5, 6, 1)
    assert torch.equal(dx == 0, y == 0)
    # as a residual of itself: x + dropout(x), written over x
    z = x.clone()
    combo.combo_dropout(z, z, z, torch.tensor(at).to(DEV), 0.2, 5, 6, 1)
    f = torch.where(y != 0, x.float() * np.float32(65536 / (65536 - 13107)), 0.0) + x.float()
    assert torch.equal(z, f.to(dtype))


def test_probabilities_at_the_ends():
    x = torch.full((9, 50), float("inf"), device=DEV)
    y = torch.empty_like(x)
    combo.combo_dropout(x, None, y, None, 1.0, 1, 2)
    assert (y == 0).all()
    x = torch.randn(9, 50, device=DEV)
    combo.combo_dropout(x, None, y, None, 0.0, 1, 2)
    assert torch.equal(x, y)


def test_share_and_independence():
    """Shares of what is kept within five deviations: over rows, columns, neighbours, sites, rounds and workers."""
    M, n, p = 2048, 512, 0.25
    x = torch.ones(M, n, device=DEV)
    masks = []
    for args, w in (((11, 0, 0), 0), ((11, 0, 1), 0), ((11, 1, 0), 0), ((12, 0, 0), 0), ((11, 0, 0), 1)):
        y = torch.empty_like(x)
        combo.combo_dropout(x, None, y, None, p, *args, first_worker=w)
        masks.append((y != 0).double())
    sd = (p * (1 - p)) ** 0.5
    q = 1 - p
    for k, a in enumerate(masks):
        assert abs(float(a.mean()) - q) < 5 * sd / (M * n) ** 0.5
        assert (a.mean(0) - q).abs().max() < 6 * sd / M ** 0.5 and (a.mean(1) - q).abs().max() < 6 * sd / n ** 0.5
        for b in masks[k + 1:]:
            assert abs(float(((a - q) * (b - q)).mean())) < 5 * sd * sd / (M * n) ** 0.5
        for s in (1, 2, 3, 4):
            assert abs(float(((a[:, s:] - q) * (a[:, :-s] - q)).mean())) < 5 * sd * sd / (M * (n - s)) ** 0.5


def test_captured_and_on_another_stream():
    x = torch.randn(700, 96, device=DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    combo.combo_dropout(x, None, y, None, 0.5, 3, 4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        combo.combo_dropout(x, None, z, None, 0.5, 3, 4)
    for _ in range(2):
        z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, z)
    z.zero_()
    torch.cuda.synchronize()
    combo.combo_dropout(x, None, z, None, 0.5, 3, 4, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, z)


def kept_rows(rows, n, p, seed, rnd, site, worker):
    """As kept(), all rows at once."""
    u = np.uint64
    with np.errstate(over="ignore"):
        z = np.arange(rows * -(-n // 4), dtype=u) ^ u(step(step(step(seed) ^ (rnd << 32 | worker)) ^ (1 << 63 | site)))
        z = z + u(0x9E3779B97F4A7C15)
        z = (z ^ (z >> u(30))) * u(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> u(27))) * u(0x94D049BB133111EB)
        z = z ^ (z >> u(31))
    return z.astype("<u8").view("<u2").reshape(rows, -(-n // 4) * 4)[:, :n] >= int(p * 65536 + 0.5)


# 148 SMs hold 4736 warps: each takes several rounds of loads, in which rows and workers change
ROUNDS = {
    "several rows": dict(n=40, each=800, workers=300, extra=8), "off 16 bytes": dict(n=37, each=500, workers=300, extra=2, skew=1),
    "parts of a row": dict(n=2500, each=50, workers=150, extra=4), "odd parts of a row": dict(n=2501, each=50, workers=150, extra=2, skew=1),
    "one worker": dict(n=200, each=40000, workers=1, extra=0), "many workers": dict(n=16, each=40, workers=8000, extra=0),
}


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", ROUNDS)
def test_several_rounds_to_a_warp(shape, dtype, residual):
    n, each, workers, extra, skew = (ROUNDS[shape].get(k, 0) for k in ("n", "each", "workers", "extra", "skew"))
    p, seed, rnd, site = 0.2, 99, 5, 3
    r = np.random.default_rng(n)
    counts = r.integers(0, 2 * each, workers) * (r.random(workers) < 0.8) if workers > 1 else [each]
    lead, behind = (3, 5) if workers > 1 else (0, 0)
    at = lead + np.concatenate([[0], np.cumsum(counts)])
    M = int(at[-1]) + behind
    g = torch.Generator().manual_seed(n)
    _, x = array(M, n, n + extra, dtype, skew, g)
    add = array(M, n, n + extra, dtype, skew, g)[1] if residual else None
    buf, y = array(M, n, n + extra, dtype, skew, g)
    before = y.clone()
    combo.combo_dropout(x, add, y, torch.tensor(at).to(DEV) if workers > 1 else None, p, seed, rnd, site)
    keep = torch.from_numpy(np.concatenate([kept_rows(int(c), n, p, seed, rnd, site, w) for w, c in enumerate(counts)])).to(DEV)
    inside = slice(int(at[0]), int(at[-1]))
    want = torch.where(keep, x[inside].float() * np.float32(65536 / (65536 - int(p * 65536 + 0.5))), 0.0)
    if residual:
        want = want + add[inside].float()
    assert torch.equal(y[inside], want.to(dtype))
    assert torch.equal(y[:lead], before[:lead]) and torch.equal(y[M - behind:], before[M - behind:])
    assert int((~buf.isnan()).sum()) == y.numel()
