"""The grouped products by pairs of CTAs, which the large bfloat16 sizes take: several stages and tiles, heights that reach
into both CTAs of a pair, ragged rows behind whole stages, operands in one copy and in a copy a block."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo
from test_gpu_grouped_linear import begin_of, f64, rows_array, run_all, weight_array

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
# more rows than a tile has, less than one 16, one more and one less than a stage and a tile, none at all
COUNTS = [0, 1, 17, 63, 64, 65, 255, 256, 257, 700, 130, 5, 31, 128, 2, 40]
PAIRS = combo.STEP_TENSOR_PAIRS


def paths(counts, n_in, n_out, dtype, odt, pad=0):
    """Which kernels the three products take at these sizes."""
    begin, M, N = begin_of(counts), sum(counts), len(counts)
    x, dy = (torch.zeros(M, n + pad, dtype=dtype, device=DEV)[:, :n] for n in (n_in, n_out))
    w = torch.zeros(N, n_out, n_in, dtype=dtype, device=DEV)
    got = []
    combo.combo_grouped_linear(x, w, torch.empty(M, n_out, dtype=odt, device=DEV), begin)
    got.append(combo.combo_last_step_path())
    combo.combo_grouped_linear_grad_input(dy, w, torch.empty(M, n_in, dtype=odt, device=DEV), begin)
    got.append(combo.combo_last_step_path())
    combo.combo_grouped_linear_grad_weight(dy, x, torch.empty(N, n_out, n_in, dtype=odt, device=DEV), begin)
    got.append(combo.combo_last_step_path())
    return got


def test_which_kernels_are_taken():
    assert paths([40, 0, 3], 24, 16, F, F) == [combo.STEP_MULTIPLY_ADD] * 3
    assert paths([40, 0, 3], 24, 16, BF, F) == [combo.STEP_TENSOR] * 3
    assert paths([40, 0, 3], 24, 16, BF, BF, pad=1) == [combo.STEP_TENSOR_THREADS] * 3
    assert paths([40, 0, 3], 25, 16, BF, BF) == [combo.STEP_TENSOR_THREADS] * 3


@pytest.mark.parametrize("odt", [BF, F])
@pytest.mark.parametrize("n_in, n_out, taken", [
    (1032, 1288, [PAIRS] * 3),                      # widths that are no multiples of 64: a copy for each block
    (1280, 1344, [PAIRS] * 3),                      # multiples of 64: one copy
    (128, 1288, [PAIRS, combo.STEP_TENSOR, PAIRS]),  # two stages; a narrow gradient of the weights
    (1290, 128 + 8, [combo.STEP_TENSOR_THREADS] * 3),
])
def test_products_match(n_in, n_out, taken, odt):
    assert paths(COUNTS, n_in, n_out, BF, odt) == taken
    run_all(COUNTS, n_in, n_out, BF, odt, seed=n_in)


@pytest.mark.parametrize("odt", [BF, F])
def test_pitches_gaps_and_rows_of_no_worker(odt):
    run_all(COUNTS, 1032, 1288, BF, odt, xp=8, yp=24, wp=16, gap=8, skew=8, seed=1, lead=13, behind=77)


@pytest.mark.parametrize("odt", [BF, F])
def test_few_rows_and_many_workers(odt):
    # tiles of 32 rows; gradients of the weights whose only stage is a ragged one
    counts = [(5 * w) % 4 for w in range(90)]
    assert paths(counts, 264, 328, BF, odt) == [PAIRS] * 3
    run_all(counts, 264, 328, BF, odt, seed=2)


@pytest.mark.parametrize("widths", [(1032, 1288), (1280, 1344)])
@pytest.mark.parametrize("odt", [BF, F])
def test_nan_stays_with_its_row_and_worker(odt, widths):
    n_in, n_out = widths
    g = torch.Generator().manual_seed(5)
    begin, M, N = begin_of(COUNTS), sum(COUNTS), len(COUNTS)
    at = np.concatenate([[0], np.cumsum(COUNTS)])
    _, x = rows_array(M, n_in, n_in, BF, g)
    _, dy = rows_array(M, n_out, n_out, BF, g)
    _, w = weight_array(N, n_out, n_in, n_in, 0, BF, g)

    def go():
        y, dx = torch.empty(M, n_out, dtype=odt, device=DEV), torch.empty(M, n_in, dtype=odt, device=DEV)
        dw = torch.empty(N, n_out, n_in, dtype=odt, device=DEV)
        combo.combo_grouped_linear(x, w, y, begin)
        combo.combo_grouped_linear_grad_input(dy, w, dx, begin)
        combo.combo_grouped_linear_grad_weight(dy, x, dw, begin)
        torch.cuda.synchronize()
        return y, dx, dw

    clean = go()
    # the last row of worker 8 (257 rows) and the first of worker 10: worker 9's rows lie between and share stages with both
    last, first = int(at[9]) - 1, int(at[10])
    x[last, n_in - 1], dy[first, n_out - 1], w[12, n_out - 1, 3] = float("nan"), float("inf"), float("nan")
    y, dx, dw = go()
    row = torch.arange(M, device=DEV)
    mine = (row >= at[12]) & (row < at[13])
    assert torch.equal(y[(row != last) & ~mine], clean[0][(row != last) & ~mine]) and torch.isnan(y[last]).all()
    assert torch.isnan(y[mine][:, n_out - 1]).all() and torch.equal(y[mine][:, :n_out - 1], clean[0][mine][:, :n_out - 1])
    assert torch.equal(dx[(row != first) & ~mine], clean[1][(row != first) & ~mine]) and not torch.isfinite(dx[first]).any()
    assert torch.isnan(dx[mine][:, 3]).all()
    other = [v for v in range(N) if v not in (8, 10)]
    assert torch.equal(dw[other], clean[2][other])
    assert torch.isnan(dw[8][:, n_in - 1]).all() and torch.equal(dw[8][:, :n_in - 1], clean[2][8][:, :n_in - 1])
    assert not torch.isfinite(dw[10][n_out - 1]).any() and torch.equal(dw[10][:n_out - 1], clean[2][10][:n_out - 1])


def test_every_time_the_same():
    a = run_all(COUNTS, 1032, 1288, BF, F, seed=3)
    b = run_all(COUNTS, 1032, 1288, BF, F, seed=3)
    for s, t in zip(a, b):
        assert np.array_equal(f64(s), f64(t))
