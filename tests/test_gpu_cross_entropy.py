"""combo_grouped_cross_entropy and its backward call against the definitions in 64 bits."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1908_07782_b200 as combo  # noqa: E402
from loss_util import DEV, U, Case  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32)]
IDS = ["f32", "bf16", "bf16-f32"]

SHAPES = {
    # the smallest, one class, one input
    "one": dict(counts=[1], n_in=1, n_out=1),
    "one class": dict(counts=[3, 2], n_in=9, n_out=1),
    "one input": dict(counts=[5, 4], n_in=1, n_out=7),
    # small classifiers, workers without rows, rows of no worker
    "classifier": dict(counts=[1] * 8, n_in=256, n_out=10),
    "ragged": dict(counts=[7, 0, 20, 1], n_in=33, n_out=13, lead=3, behind=2, mean=False),
    "masked": dict(counts=[40, 9, 0, 64], n_in=64, n_out=21, keep=0.3),
    # larger than a tile in each direction, odd widths
    "wide": dict(counts=[130, 300], n_in=200, n_out=700),
    "odd": dict(counts=[129, 65, 0, 257], n_in=77, n_out=301, keep=0.6, mean=False),
    "classes": dict(counts=[70, 3], n_in=136, n_out=2500),
    "long": dict(counts=[1100], n_in=520, n_out=513, keep=0.9),
    "deep": dict(counts=[66], n_in=2300, n_out=260),
    "many workers": dict(counts=[k % 4 for k in range(300)], n_in=72, n_out=300),
    # places and pitches: 16-byte ones that are not dense, and others
    "pitches": dict(counts=[33, 140], n_in=128, n_out=384, xp=8, wp=16, gap=64),
    "off 16 bytes": dict(counts=[33, 140], n_in=128, n_out=384, xp=3, wp=1, gap=5, skew=1),
}


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_values_and_gradients(shape, types):
    c = Case(dtype=types[0], out=types[1], seed=len(shape), **SHAPES[shape])
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    outside = c.dx[~c.inside].clone()
    c.backward(lse)
    c.check_backward(lse)
    assert torch.equal(c.dx[~c.inside], outside)
    # nothing between the rows, nor between the workers' weights
    for buf, t in ((c.dx_buf, c.dx), (c.dw_buf, c.dw)):
        assert int((~buf.isnan()).sum()) == t.numel()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_row_has_a_label(dtype):
    c = Case([5, 0, 70], 40, 300, dtype, keep=0.0)
    c.forward()
    assert (c.loss == 0).all() and (c.lse == 0).all()
    c.backward(c.lse)
    assert (c.dx == 0).all() and (c.dw == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows(dtype):
    c = Case([0, 0], 40, 300, dtype)
    c.forward()
    c.backward(c.lse)
    assert (c.dw == 0).all()


@pytest.mark.parametrize("n_out", [20, 600])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_logits(dtype, n_out):
    """Logits of a thousand and more: only differences are exponentiated."""
    c = Case([40, 130], 64, n_out, dtype, spread=400.0)
    c.forward()
    c.check_forward()
    assert float(c.lse.max()) > 500
    lse = c.lse.clone()
    c.backward(lse)
    c.check_backward(lse)


@pytest.mark.parametrize("n_out", [12, 520])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_and_infinity_stay_in_their_row_and_worker(dtype, n_out):
    c = Case([20, 150, 9], 48, n_out, dtype)
    good = Case([20, 150, 9], 48, n_out, dtype)
    for k in (c, good):
        k.forward()
    good.backward(good.lse)
    c.x[25, 3] = float("nan")
    c.x[120, 5] = float("inf")
    c.w[2, 7, 1] = float("nan")
    c.forward()
    bad = torch.zeros(c.M, dtype=torch.bool, device=DEV)
    bad[[25, 120]] = True
    bad[170:] = True
    assert c.loss[bad].isnan().all() and torch.equal(c.loss[~bad], good.loss[~bad])
    c.backward(c.lse)
    assert c.dx[bad].isnan().any(1).all() and torch.equal(c.dx[~bad], good.dx[~bad])
    assert torch.equal(c.dw[0], good.dw[0]) and c.dw[1].isnan().any() and c.dw[2].isnan().any()


def test_a_class_at_minus_infinity_is_none():
    """Weights of -inf against a positive input: the class has probability zero."""
    c = Case([30], 16, 400, BF16)
    c.x[:, 0] = 1.0
    c.w[0, 399, 0] = float("-inf")
    c.labels[:] = 5
    c.forward()
    w = c.w[0, :399].double()
    want = torch.logsumexp(c.x.double() @ w.T, 1)
    assert (c.lse.double() - want).abs().max() < 1e-4
    assert not c.loss.isnan().any()


@pytest.mark.parametrize("counts,n_in,n_out", [([6, 0, 9], 24, 11), ([40, 130], 96, 520)])
def test_gradients_against_differences(counts, n_in, n_out):
    c = Case(counts, n_in, n_out, F32, mean=False, keep=0.7)
    c.forward()
    c.backward(c.lse)
    g = torch.Generator().manual_seed(3)
    ux, uw = torch.randn(c.M, n_in, generator=g).to(DEV), torch.randn(c.w.shape, generator=g).to(DEV) / n_in ** 0.5
    x0, w0, h = c.x.clone(), c.w.clone(), 2.0 ** -7
    for dx, dw in ((ux, None), (None, uw)):
        losses = []
        for sign in (1, -1):
            c.x.copy_(x0 if dx is None else x0 + sign * h * dx)
            c.w.copy_(w0 if dw is None else w0 + sign * h * dw)
            c.forward()
            losses.append(c.loss.double())
        c.x.copy_(x0)
        c.w.copy_(w0)
        got = ((losses[0] - losses[1]) * c.row_grad.double() * c.has).sum() / (2 * h)
        want = (c.dx.double() * dx.double())[c.has].sum() if dw is None else (c.dw.double() * dw.double()).sum()
        # the third derivative of a log-sum-exp is a third central moment, R^3 q (1 - q) (1 - 2 q) for two values R apart, at most
        # R^3 / (6 sqrt(3)) over the range R of the logits' change; float inputs moved by h are off by half a unit; the losses'
        # own error
        tol = 0.0
        for w in range(c.N):
            rows, x, wt, z, dz = c.logits(w)
            if len(rows):
                move = dx[rows].double() @ wt.T if dw is None else x @ dw[w].double().T
                spread = move.max(1).values - move.min(1).values
                error = 4 * dz.max(1).values + (200 + c.V / 8) * U * 2
                tol += float((c.row_grad[rows].double().abs() * (h * h / 6 * spread ** 3 / (6 * 3 ** 0.5) + error / h)).sum())
        assert abs(float(got - want)) <= tol and tol < 0.25 * abs(float(want)) + 1.0


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_same_bits_from_run_to_run_and_from_a_graph(types):
    c = Case([300, 20, 0, 410], 136, 1000, types[0], types[1], keep=0.8)
    f, b = c.scratch(False), c.scratch(True)
    c.forward(f)
    c.backward(c.lse, b)
    first = [t.clone() for t in (c.loss, c.lse, c.dx, c.dw)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.forward(f)
            c.backward(c.lse, b)
    for _ in range(3):
        for t in (c.loss, c.lse, c.dx, c.dw):
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, k) for t, k in zip((c.loss, c.lse, c.dx, c.dw), first))


def test_two_calls_at_once():
    a, b = Case([500, 300], 264, 1500, BF16, seed=1), Case([200, 610], 264, 1500, BF16, seed=2)
    for c in (a, b):
        c.forward()
        c.backward(c.lse)
    torch.cuda.synchronize()
    want = [t.clone() for c in (a, b) for t in (c.loss, c.dx, c.dw)]
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    pa, pb = [(c.scratch(False), c.scratch(True)) for c in (a, b)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, p in ((a, sa, pa), (b, sb, pb)):
            with torch.cuda.stream(s):
                c.forward(p[0])
                c.backward(c.lse, p[1])
    torch.cuda.synchronize()
    assert all(torch.equal(t, k) for t, k in zip([t for c in (a, b) for t in (c.loss, c.dx, c.dw)], want))


def test_a_view_beside_the_input():
    """x and dx as columns of one array."""
    c = Case([40, 30], 32, 300, F32)
    c.backward(c.exact_lse())
    want = c.dx.clone()
    wide = torch.zeros(c.M, 64, device=DEV)
    wide[:, :32] = c.x
    combo.combo_grouped_cross_entropy_backward(wide[:, :32], c.w, c.labels, c.exact_lse(), None, wide[:, 32:], c.dw, c.begin, c.scratch(True))
    assert torch.equal(wide[:, 32:], want)


# Pairs of CTAs in both directions: eight warps for the results, several tiles along the inputs, workers' ends inside a pair.
BY_PAIRS = {
    "dense": dict(counts=[300, 0, 200], n_in=776, n_out=1500, keep=0.6),
    "factors": dict(counts=[300, 0, 200], n_in=776, n_out=1500, keep=0.6, mean=False),
    "off 16 bytes": dict(counts=[300, 0, 200], n_in=776, n_out=1500, keep=0.6, xp=3, wp=1, skew=1),
    "ends inside 16 bytes": dict(counts=[150, 290], n_in=773, n_out=1501, xp=3, wp=3, gap=8, mean=False),
}


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", BY_PAIRS)
def test_values_and_gradients_by_pairs(shape, types):
    c = Case(dtype=types[0], out=types[1], seed=len(shape), **BY_PAIRS[shape])
    c.forward()
    assert combo.combo_last_step_path() == combo.STEP_TENSOR_PAIRS
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_TENSOR_PAIRS
    c.check_backward(lse)
    for buf, t in ((c.dx_buf, c.dx), (c.dw_buf, c.dw)):
        assert int((~buf.isnan()).sum()) == t.numel()


@pytest.mark.parametrize("n_out,path", [(13, combo.STEP_MULTIPLY_ADD), (301, combo.STEP_TENSOR)])
@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_widths_that_end_inside_16_bytes(types, n_out, path):
    """Places, pitches and strides on 16 bytes, widths that are not."""
    c = Case([129, 65, 0, 257], 77, n_out, types[0], types[1], keep=0.6, mean=False, xp=3, wp=3, gap=8)
    c.forward()
    assert combo.combo_last_step_path() == path
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == path
    c.check_backward(lse)
    for buf, t in ((c.dx_buf, c.dx), (c.dw_buf, c.dw)):
        assert int((~buf.isnan()).sum()) == t.numel()


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_more_workers_than_threads_in_few_multiply_adds(types):
    c = Case([k % 3 for k in range(700)], 32, 10, types[0], types[1], lead=1, behind=2, keep=0.8)
    c.forward()
    assert combo.combo_last_step_path() == combo.STEP_MULTIPLY_ADD
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_MULTIPLY_ADD
    c.check_backward(lse)


@pytest.mark.parametrize("mean", [True, False])
@pytest.mark.parametrize("counts,n_in,n_out", [([40, 1, 9], 48, 400), ([60, 33], 32, 600), ([64] * 40, 64, 20)])
def test_float_gradients_of_bfloat16_rows_have_float_precision(counts, n_in, n_out, mean):
    """Seen over a worker's gradients as a whole: d enters a float dW to 24 bits."""
    c = Case(counts, n_in, n_out, BF16, F32, mean=mean)
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_TENSOR
    for w in range(c.N):
        rows, x, wt, z, dz = c.logits(w)
        g = torch.full((len(rows), 1), 1.0 / len(rows), dtype=torch.float64, device=DEV) if mean else c.row_grad[rows].double()[:, None]
        p = torch.exp(z - lse[rows].double()[:, None])
        hot = torch.zeros_like(p).scatter_(1, c.labels[rows, None], 1.0)
        want = ((p - hot) * g).T @ x
        error = float((c.dw[w].double() - want).norm() / want.norm())
        # the tensor cores truncate when they add 16 products: logits, of 1.5 on average, by n_in / 16 units of 2 U, the sums over the
        # rows by as many as there are sixteens; an exponential is off by 4 U, d by 3 more, what its three planes leave by one
        assert error <= (1.5 * 2 * (n_in / 16 + 1) + 8 + 2 * (len(rows) / 16 + 1)) * U, error / U


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("counts,n_in,n_out", [([300, 200], 5000, 120), ([300, 1], 4500, 250), ([600], 530, 1024)])
def test_pairs_with_few_classes(counts, n_in, n_out, types):
    """One or two tiles along the classes, less than a pair's height of them."""
    c = Case(counts, n_in, n_out, types[0], types[1], keep=0.9, mean=False)
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_TENSOR_PAIRS
    c.check_backward(lse)


@pytest.mark.parametrize("large", [2.0 ** 12, 2.0 ** 20, 2.0 ** 30])
@pytest.mark.parametrize("counts,n_in,n_out", [([6, 9], 24, 11), ([40, 130], 96, 520), ([300, 200], 600, 700)])
def test_one_input_far_larger_than_the_others(counts, n_in, n_out, large):
    """Floats: an input that is large where its weights are nothing or small, and a class with one large weight."""
    c = Case(counts, n_in, n_out, F32, mean=False, keep=0.8)
    c.x[:, 5] *= large
    c.w[:, :, 5] = 0.0
    c.w[0, 3, 7] *= large
    c.x[:, 7] /= large
    c.w[:, 4, 5] = 0.5 / large
    c.forward()
    few = combo.combo_last_step_path() == combo.STEP_MULTIPLY_ADD
    for w in range(c.N):
        rows, x, wt, z, dz = c.logits(w)
        # two planes of float16 keep 22 bits of a value, or 2^-39 of the largest of its row or class if that is more: an error of half
        # of float16's least number, 2^-25, in units that take the largest to at least 2^14
        if not few:
            dz = dz + 2.0 ** -39 * (x.abs().amax(1)[:, None] * wt.abs().sum(1) + x.abs().sum(1)[:, None] * wt.abs().amax(1)) + \
                c.K * 2.0 ** -78 * x.abs().amax(1)[:, None] * wt.abs().amax(1)
        lse, own = torch.logsumexp(z, 1), z.gather(1, c.labels[rows, None])[:, 0]
        tol = dz.max(1).values + (200 + c.V / 8) * U + 4 * U * (lse.abs() + z.max(1).values.abs())
        assert ((c.lse[rows].double() - lse).abs() <= tol).all()
        assert ((c.loss[rows].double() - (lse - own)).abs() <= tol + dz.max(1).values + 2 * U * own.abs()).all()
    # backward keeps 24 bits of every value
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


@pytest.mark.parametrize("dtype,counts,n_in,n_out,mean", [(F32, [1800, 1750, 1790], 128, 18, False), (F32, [700, 800, 650], 120, 8, True),
                                                          (BF16, [1200, 300, 900], 1408, 14, True), (BF16, [2, 5, 3], 1304, 65, True)])
def test_gradients_of_few_classes_are_as_exact_as_32_bit_arithmetic(dtype, counts, n_in, n_out, mean):
    """Errors over all of a float gradient: within 1.5 times those of the same formula in 32-bit torch arithmetic, or 16 units."""
    c = Case(counts, n_in, n_out, dtype, F32, mean=mean)
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_TENSOR
    got, want, plain = [], [], []
    for w, (a, b) in enumerate(c.spans):
        for t, to in ((torch.float64, want), (torch.float32, plain)):
            x, wt = c.x[a:b].to(t), c.w[w].to(t)
            g = torch.full((b - a, 1), 1.0 / (b - a), dtype=t, device=DEV) if mean else c.row_grad[a:b, None].to(t)
            d = torch.exp(x @ wt.T - lse[a:b, None].to(t))
            d.scatter_add_(1, c.labels[a:b, None], torch.full((b - a, 1), -1.0, dtype=t, device=DEV))
            to.append((d * g).T @ x)
        got.append(c.dw[w])
    got, want, plain = (torch.stack(t).double() for t in (got, want, plain))
    error, allowed = float((got - want).norm() / want.norm()), float((plain - want).norm() / want.norm())
    assert error <= max(16 * U, 1.5 * allowed), (error, allowed)


@pytest.mark.parametrize("counts,n_in,n_out", [([1] * 9, 64, 700), ([2, 1, 40, 0, 3], 200, 1500), ([70, 60], 333, 264), ([128] * 3, 72, 2000)])
def test_bfloat16_gradients_of_few_rows_are_rounded_once(counts, n_in, n_out):
    """d enters a bfloat16 dW of few rows a worker to 16 bits, so that the last rounding is nearly all that it is off by."""
    c = Case(counts, n_in, n_out, BF16, BF16, mean=False, keep=0.9)
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == combo.STEP_TENSOR
    for w in range(c.N):
        rows, x, wt, z, dz = c.logits(w)
        e, g = lse[rows].double()[:, None], c.row_grad[rows].double()[:, None]
        p = torch.exp(z - e)
        hot = torch.zeros_like(p).scatter_(1, c.labels[rows, None], 1.0)
        d = (p - hot) * g
        # as in Case.check_backward, but for d's own rounding: 2^-16 of it, after two planes of half a step of 2^-8 each
        dd = g.abs() * (p * (dz + (60 + 4 * (z.abs() + e.abs())) * U) + 2 * U * (p + hot) + 2.0 ** -126) + 2.0 ** -16 * d.abs()
        Case.near(c.dw[w], d.T @ x, dd.T @ x.abs() + 2 * (len(rows) + 4) * U * (d.abs().T @ x.abs()), 2.0 ** -8, "dw of worker %d" % w)
