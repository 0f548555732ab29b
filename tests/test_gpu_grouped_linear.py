"""combo_grouped_linear and its two gradients against the products in 64 bits."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)]


def half_ulp_bf16(v):
    return 0.5 * 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 7)


def f64(t):
    return t.detach().cpu().double().numpy()


def rows_array(M, width, pitch, dtype, g, skew=0, fill=None):
    """[M, width] with `pitch` elements between rows, `skew` before the first; NaN everywhere else."""
    buf = torch.full((skew + M * pitch + 16,), float("nan"), dtype=dtype, device=DEV)
    t = buf[skew:skew + M * pitch].view(M, pitch)[:, :width]
    t.copy_(torch.randn(M, width, generator=g) if fill is None else torch.full((M, width), fill))
    return buf, t


def weight_array(N, n_out, n_in, pitch, gap, dtype, g, skew=0, fill=None):
    stride = n_out * pitch + gap
    buf = torch.full((skew + N * stride + 16,), float("nan"), dtype=dtype, device=DEV)
    t = buf[skew:].as_strided((N, n_out, n_in), (stride, pitch, 1), skew)
    t.copy_(torch.randn(N, n_out, n_in, generator=g) if fill is None else torch.full((N, n_out, n_in), fill))
    return buf, t


def begin_of(counts, lead=0):
    return torch.tensor(lead + np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)).to(DEV)


def close(got, want, size, depth, odt):
    """Products are exact to half a unit and `depth` of them are added: each addition errs by a unit in the last place
    at most (tensor cores truncate), relative to the sum of the magnitudes; the result is rounded once."""
    tol = 2 * (depth + 4) * U * size
    if odt == torch.bfloat16:
        tol = tol + half_ulp_bf16(np.abs(want) + tol)
    bad = np.abs(got - want) > tol
    assert not bad.any() and not np.isnan(got).any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) / (tol + 1e-30))))


def run_all(counts, n_in, n_out, dtype, odt, xp=0, yp=0, wp=0, gap=0, skew=0, seed=0, lead=0, behind=0):
    g = torch.Generator().manual_seed(seed)
    N, M = len(counts), lead + sum(counts) + behind
    begin = begin_of(counts, lead)
    spans = [(int(a), int(b)) for a, b in zip(begin[:-1].cpu(), begin[1:].cpu())]
    _, x = rows_array(M, n_in, n_in + xp, dtype, g, skew)
    _, dy = rows_array(M, n_out, n_out + yp, dtype, g, skew)
    _, w = weight_array(N, n_out, n_in, n_in + wp, gap, dtype, g, skew)
    if lead:
        x[:lead], dy[:lead] = float("nan"), float("nan")
    if behind:
        x[-behind:], dy[-behind:] = float("nan"), float("nan")
    ybuf, y = rows_array(M, n_out, n_out + yp, odt, g, skew, fill=3.0)
    dxbuf, dx = rows_array(M, n_in, n_in + xp, odt, g, skew, fill=3.0)
    dwbuf, dw = weight_array(N, n_out, n_in, n_in + wp, gap, odt, g, skew, fill=3.0)
    kept = [torch.isnan(b).sum() for b in (ybuf, dxbuf, dwbuf)]
    combo.combo_grouped_linear(x, w, y, begin)
    combo.combo_grouped_linear_grad_input(dy, w, dx, begin)
    combo.combo_grouped_linear_grad_weight(dy, x, dw, begin)
    torch.cuda.synchronize()
    combo.combo_device_status()
    X, DY, W, Y, DX, DW = (f64(t) for t in (x, dy, w, y, dx, dw))
    for v, (a, b) in enumerate(spans):
        close(Y[a:b], X[a:b] @ W[v].T, np.abs(X[a:b]) @ np.abs(W[v]).T, n_in, odt)
        close(DX[a:b], DY[a:b] @ W[v], np.abs(DY[a:b]) @ np.abs(W[v]), n_out, odt)
        close(DW[v], DY[a:b].T @ X[a:b], np.abs(DY[a:b]).T @ np.abs(X[a:b]), b - a, odt)
    # rows of no worker, and everything between rows and behind them, are as they were
    assert (Y[:lead] == 3).all() and (DX[:lead] == 3).all()
    if behind:
        assert (Y[-behind:] == 3).all() and (DX[-behind:] == 3).all()
    assert kept == [torch.isnan(b).sum() for b in (ybuf, dxbuf, dwbuf)], "written outside the results"
    return y, dx, dw


SHAPES = [
    # rows of the workers, n_in, n_out
    ([1], 1, 1),
    ([1], 8, 8),
    ([0, 1, 0, 3], 24, 10),
    ([5, 2], 33, 17),
    ([1] * 9, 64, 128),
    ([127, 128, 129], 64, 136),
    ([300, 1, 0, 255, 257], 72, 264),
    ([64] * 3, 512, 256),
    ([31, 33, 0, 0, 16, 15, 17, 32], 200, 120),
    ([700], 1000, 96),
    ([65, 63, 64, 1], 128, 1000),
    ([0, 0], 16, 16),
    ([3] * 300, 16, 24),
]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("k", range(len(SHAPES)))
def test_products_match(k, types):
    counts, n_in, n_out = SHAPES[k]
    run_all(counts, n_in, n_out, *types, seed=k)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("k", range(2, len(SHAPES), 2))
def test_pitches_and_gaps(k, types):
    counts, n_in, n_out = SHAPES[k]
    run_all(counts, n_in, n_out, *types, xp=8, yp=16, wp=8, gap=24, skew=8, seed=k)      # still multiples of 16 bytes or not, by the width
    run_all(counts, n_in, n_out, *types, xp=3, yp=1, wp=5, gap=7, skew=1, seed=k)


@pytest.mark.parametrize("types", TYPES)
def test_rows_of_no_worker(types):
    run_all([40, 0, 130, 7], 96, 80, *types, lead=11, behind=5)


@pytest.mark.parametrize("types", TYPES)
def test_larger(types):
    run_all([500, 1100, 0, 731], 520, 776, *types, seed=3)


@pytest.mark.parametrize("widths", [(72, 88), (71, 89)])
@pytest.mark.parametrize("types", TYPES)
def test_nan_stays_with_its_row_and_worker(types, widths):
    dtype, odt = types
    g = torch.Generator().manual_seed(5)
    counts, (n_in, n_out) = [70, 60, 130], widths
    begin = begin_of(counts)
    _, x = rows_array(260, n_in, n_in, dtype, g)
    _, dy = rows_array(260, n_out, n_out, dtype, g)
    _, w = weight_array(3, n_out, n_in, n_in, 0, dtype, g)
    outs = lambda: (torch.empty(260, n_out, dtype=odt, device=DEV), torch.empty(260, n_in, dtype=odt, device=DEV),  # noqa: E731
                    torch.empty(3, n_out, n_in, dtype=odt, device=DEV))

    def go(y, dx, dw):
        combo.combo_grouped_linear(x, w, y, begin)
        combo.combo_grouped_linear_grad_input(dy, w, dx, begin)
        combo.combo_grouped_linear_grad_weight(dy, x, dw, begin)
        torch.cuda.synchronize()
        return y, dx, dw

    clean = go(*outs())
    x[69, 5], dy[130, 7], w[2, 3, 4] = float("nan"), float("inf"), float("nan")
    y, dx, dw = go(*outs())
    own = torch.arange(260, device=DEV)
    good = (own != 69) & (own < 130)
    assert torch.equal(y[good], clean[0][good]) and torch.isnan(y[69]).all()
    assert torch.isnan(y[130:, 3]).all()
    assert torch.equal(dx[:130], clean[1][:130])
    assert torch.equal(dw[1], clean[2][1])                    # its neighbours' rows share tiles with it
    assert torch.isnan(dw[0][:, 5]).all() and not torch.isnan(dw[0][:, 6]).any()
    assert not torch.isfinite(dw[2][7]).any() and torch.isfinite(dw[2][8]).all()


def test_same_result_on_another_stream_and_every_time():
    first = run_all([300, 77], 256, 384, torch.bfloat16, torch.bfloat16, seed=9)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = run_all([300, 77], 256, 384, torch.bfloat16, torch.bfloat16, seed=9)
    for a, b in zip(first, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_against_differences(dtype):
    # loss = sum(dy * y) is linear in x and in w: its difference along a direction is exact in 64 bits
    g = torch.Generator().manual_seed(6)
    counts, n_in, n_out = [33, 0, 20], 40, 56
    begin = begin_of(counts)
    _, x = rows_array(53, n_in, n_in, dtype, g)
    _, dy = rows_array(53, n_out, n_out, dtype, g)
    _, w = weight_array(3, n_out, n_in, n_in, 0, dtype, g)
    dx = torch.empty(53, n_in, device=DEV)
    dw = torch.empty(3, n_out, n_in, device=DEV)
    combo.combo_grouped_linear_grad_input(dy, w, dx, begin)
    combo.combo_grouped_linear_grad_weight(dy, x, dw, begin)
    X, DY, W = f64(x), f64(dy), f64(w)
    spans = [(0, 33), (33, 33), (33, 53)]

    def loss(X, W):
        return sum(float((DY[a:b] * (X[a:b] @ W[v].T)).sum()) for v, (a, b) in enumerate(spans))

    r = np.random.RandomState(1)
    for vx, vw, got in ((r.randn(*X.shape), np.zeros_like(W), f64(dx)), (np.zeros_like(X), r.randn(*W.shape), f64(dw))):
        diff = (loss(X + 0.5 * vx, W + 0.5 * vw) - loss(X - 0.5 * vx, W - 0.5 * vw))
        v = vx if vx.any() else vw
        # every gradient is off by at most 2 (n + 4) U of its magnitudes' sum, 60 terms at most, each about 1
        assert abs(diff - float((got * v).sum())) <= 2 * 64 * U * 64 * float(np.abs(v).sum())


def test_weights_at_large_offsets():
    # the last worker's weights lie beyond 2^32 bytes
    N, P = 5, 500_000_000
    flat = torch.zeros(N * P, dtype=torch.bfloat16, device=DEV).view(N, P)
    w = flat[:, 1000:1000 + 64 * 128].unflatten(1, (64, 128))
    w[4] = 1.0
    w[3] = 2.0
    x = torch.ones(20, 128, dtype=torch.bfloat16, device=DEV)
    y = torch.empty(20, 64, dtype=torch.bfloat16, device=DEV)
    begin = begin_of([4] * 5)
    combo.combo_grouped_linear(x, w, y, begin)
    assert (y[16:] == 128).all() and (y[12:16] == 256).all() and (y[:12] == 0).all()
    combo.combo_grouped_linear_grad_weight(y, x, w, begin)
    assert (w[4] == 512).all() and (w[3] == 1024).all() and (w[:3] == 0).all()
    assert (flat[4, :1000] == 0).all() and (flat[4, 1000 + 64 * 128:1000 + 64 * 128 + 1000] == 0).all()


def test_refusals():
    x = torch.zeros(10, 16, device=DEV)
    w = torch.zeros(2, 8, 16, device=DEV)
    y = torch.zeros(10, 8, device=DEV)
    begin = begin_of([4, 6])
    lib = combo.load()

    def call(**kw):
        a = dict(x=x.data_ptr(), xp=16, w=w.data_ptr(), wp=16, ws=128, y=y.data_ptr(), yp=8, eb=4, ob=4, begin=begin.data_ptr(),
                 N=2, M=10, n_in=16, n_out=8)
        a.update(kw)
        return lib.combo_grouped_linear(a["x"], a["xp"], a["w"], a["wp"], a["ws"], a["y"], a["yp"], a["eb"], a["ob"], a["begin"],
                                        a["N"], a["M"], a["n_in"], a["n_out"], None)

    assert call() == 0
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(begin=None), dict(eb=2, ob=8), dict(eb=4, ob=2), dict(eb=8, ob=8),
               dict(N=0), dict(N=8193), dict(M=-1), dict(n_in=0), dict(n_out=0), dict(xp=15), dict(yp=7), dict(wp=15),
               dict(ws=127), dict(x=x.data_ptr() + 2), dict(begin=begin.data_ptr() + 4), dict(n_in=(1 << 20) + 1)):
        assert call(**kw) == 1, kw
    assert call(y=x.data_ptr()) == 2 and call(y=w.data_ptr(), M=10) == 2
    assert call(M=0, x=None, y=None) == 0
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        combo.combo_grouped_linear(x, w, y[:9], begin)
    with pytest.raises(ValueError):
        combo.combo_grouped_linear(x, w.transpose(1, 2), y, begin)
    with pytest.raises(ValueError):
        combo.combo_grouped_linear(x.bfloat16(), w, y, begin)
    with pytest.raises(ValueError):
        combo.combo_grouped_linear(x, w, y, begin.int())
    with pytest.raises(ValueError):
        combo.combo_grouped_linear(x.double(), w.double(), y, begin)
