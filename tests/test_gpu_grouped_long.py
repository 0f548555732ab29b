"""Grouped products whose sums are so long that they are cut into parts (more than 4096 values), between others that are not."""
import pytest
import torch

import paper_1908_07782_b200 as combo
from test_gpu_grouped_linear import begin_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
ULP = 2.0 ** -23
PART = 4096


def values(g, sign, *shape):
    v = torch.rand(*shape, generator=g, device=DEV) + 0.5 if sign else torch.randn(*shape, generator=g, device=DEV)
    return v.to(BF)


def check(got, a, b):
    """got [i, j] against sum_r a [i, r] b [j, r] in 64 bits.  Of a part, n of 16 products at a time: the accumulator grows
    evenly where all terms have one sign, so that the truncations, a unit each, come to n / 2 units of the part (and to no more
    than that of the sum of the magnitudes, whatever the signs); 16 more for the products of a step and the last one's.
    The parts are added with half a unit each, evenly growing again.  Rounded once."""
    a, b = a.double(), b.double()
    want, size = a @ b.T, a.abs() @ b.abs().T
    r = a.shape[1]
    parts = -(-r // PART)
    tol = ((min(r, PART) / 16 / 2 + 16) + parts / 4 + 1) * ULP * size
    if got.dtype == BF:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    off = (got.double() - want).abs()
    assert (off <= tol).all(), float((off / (size * ULP)).max())


def forward(g, sign, counts, n_in, n_out, odt, grad):
    """The forward product, or (`grad`) the gradient of the rows, whose sums run over n_in."""
    begin, M, N = begin_of(counts), sum(counts), len(counts)
    x = values(g, sign, M, n_in)
    w = values(g, sign, N, n_in, n_out) if grad else values(g, sign, N, n_out, n_in)
    y = torch.full((M, n_out), 7.0, dtype=odt, device=DEV)
    (combo.combo_grouped_linear_grad_input if grad else combo.combo_grouped_linear)(x, w, y, begin)
    taken = combo.combo_last_step_path()
    at = 0
    for v, n in enumerate(counts):
        if n:
            check(y[at:at + n], x[at:at + n], w[v].T if grad else w[v])
        at += n
    combo.combo_device_status()
    return taken


def weights(g, sign, counts, n_in, n_out, odt):
    begin, M, N = begin_of(counts), sum(counts), len(counts)
    x, dy = values(g, sign, M, n_in), values(g, sign, M, n_out)
    dw = torch.full((N, n_out, n_in), 7.0, dtype=odt, device=DEV)
    combo.combo_grouped_linear_grad_weight(dy, x, dw, begin)
    taken = combo.combo_last_step_path()
    at = 0
    for v, n in enumerate(counts):
        if n:
            check(dw[v], dy[at:at + n].T, x[at:at + n].T)
        else:
            assert (dw[v] == 0).all()
        at += n
    combo.combo_device_status()
    return taken


@pytest.fixture()
def g():
    return torch.Generator(device=DEV).manual_seed(11)


@pytest.mark.parametrize("sign", [True, False])
@pytest.mark.parametrize("odt", [BF, F])
@pytest.mark.parametrize("n_in, n_out", [(128, 128), (200, 136), (129, 64)])
def test_gradient_of_the_weights(g, sign, odt, n_in, n_out):
    taken = weights(g, sign, [65_536 + 37, 0, 4096, 4097, 100, 8192], n_in, n_out, odt)
    assert taken == (combo.STEP_TENSOR_THREADS if n_in % 8 else combo.STEP_TENSOR)


@pytest.mark.parametrize("odt", [BF, F])
def test_gradient_of_the_weights_by_pairs(g, odt):
    # four tiles a worker: a pair of CTAs meets whole sums, sums in parts and none in every order
    lengths = [5000, 0, 64, 4096, 4097, 8193, 100, 12_288, 1, 4160, 3000, 9000, 4095]
    counts = [lengths[(7 * w) % 13] for w in range(60)]
    assert weights(g, True, counts, 256, 1024, odt) == combo.STEP_TENSOR_PAIRS


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("odt", [BF, F])
@pytest.mark.parametrize("n_in", [4096, 4104, 10_008, 10_001])
def test_products_of_wide_rows(g, odt, n_in, grad):
    few = forward(g, True, [3, 0, 40], n_in, 136, odt, grad)
    # by pairs, several tiles for each
    many = forward(g, True, [300, 1, 0, 257, 64, 90, 5, 33, 16, 255], n_in, 2048, odt, grad)
    # the gradient's weights have rows of 136 and 2048: only its own rows are off 16-byte boundaries
    assert (few, many) == ((combo.STEP_TENSOR_THREADS,) * 2 if n_in == 10_001 else (combo.STEP_TENSOR, combo.STEP_TENSOR_PAIRS))


def test_every_length_about_a_part(g):
    for r in (4032, 4033, 4095, 4096, 4097, 4111, 4112, 4113, 4159, 4160, 4161, 8191, 8192, 8193):
        weights(g, True, [r], 64, 64, F)


def test_a_very_long_sum(g):
    x = values(g, True, 1 << 20, 64)
    dw = torch.empty(1, 64, 64, device=DEV)
    combo.combo_grouped_linear_grad_weight(x, x, dw, begin_of([1 << 20]))
    check(dw[0], x.T, x.T)


def test_nan_and_infinity(g):
    n = 9000
    x, dy = values(g, False, n, 64), values(g, False, n, 64)
    x[100, 3], x[8500, 5], dy[4096, 7] = float("nan"), float("inf"), float("nan")
    dw = torch.empty(1, 64, 64, device=DEV)
    combo.combo_grouped_linear_grad_weight(dy, x, dw, begin_of([n]))
    bad = ~torch.isfinite(dw[0])
    want = torch.zeros(64, 64, dtype=torch.bool, device=DEV)
    want[:, 3], want[:, 5], want[7] = True, True, True
    assert torch.equal(bad, want)
