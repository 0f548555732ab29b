"""The loss of rows whose label's class leads by far: it goes to zero and is never below, however large the logits are."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1908_07782_b200 as combo  # noqa: E402
from loss_util import DEV, U, Case  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def confident(counts, n_in, n_out, dtype, lead, offset):
    """Rows with one input of 1, so that logits are weights, which either type holds: the label's `offset`, the others' `lead` to
    `lead` + 24 below."""
    c = Case(counts, n_in, n_out, dtype)
    g = torch.Generator().manual_seed(n_out)
    pick = torch.arange(c.M) % n_in
    label = (pick * 7 + 3) % n_out
    w = offset - lead - torch.randint(0, 25, c.w.shape, generator=g).double()
    w[:, (torch.arange(n_in) * 7 + 3) % n_out, torch.arange(n_in)] = offset
    c.x.zero_()
    c.x[torch.arange(c.M), pick] = 1.0
    c.w.copy_(w)
    assert torch.equal(c.w.double().cpu(), w)
    c.labels.copy_(label)
    return c


@pytest.mark.parametrize("offset", [20.0, -30.0, 120.0, 250.0])
@pytest.mark.parametrize("counts,n_in,n_out,path", [([3, 1, 20], 64, 10, combo.STEP_MULTIPLY_ADD), ([40, 130], 64, 700, combo.STEP_TENSOR),
                                                    ([40, 130], 600, 2000, combo.STEP_TENSOR), ([300, 200], 600, 700, combo.STEP_TENSOR_PAIRS)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_losses_of_large_logits(dtype, counts, n_in, n_out, path, offset):
    c = confident(counts, n_in, n_out, dtype, 10.0, offset)
    c.forward()
    assert combo.combo_last_step_path() == path
    for w, (a, b) in enumerate(c.spans):
        z = c.x[a:b].double() @ c.w[w].double().T
        own = z.gather(1, c.labels[a:b, None])
        # what the other classes add to 1, in 64 bits without cancellation
        rest = (torch.exp(z - own).sum(1) - 1.0).clamp(min=0.0)
        want, lse = torch.log1p(rest), torch.logsumexp(z, 1)
        assert (want > 1e-9).any() and (want < 0.1).all()
        # The differences of these logits are exact.  An exponential's argument is off by two roundings of some 50 and its result by
        # a few units, the others' sum by as many units as it has terms.  A sum that holds the 1 is rounded by at most U (1 + rest) at
        # every addition: 32 of a thread's 128 classes and 2 of its four sums, 8 of its pieces at a time (there are no more than 32
        # here for four warps) and 32 of the warps' (few multiply-adds: 32 joins of two roundings); then the logarithm and the last
        # addition.
        tol = rest * (200 + n_out / 8) * U + 76 * U * (1 + rest)
        got = c.loss[a:b].double()
        assert (got >= 0).all() and ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())
        assert ((c.lse[a:b].double() - lse).abs() <= tol + 2 * U * lse.abs()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,n_in,n_out", [([9, 30], 40, 20), ([40, 130], 64, 700), ([400, 300], 600, 1500)])
def test_saturated_rows_have_no_loss(counts, n_in, n_out, dtype):
    """Logits of hundreds: where the label leads by 40, one plus the others is one."""
    c = Case(counts, n_in, n_out, dtype, spread=300.0)
    for w, (a, b) in enumerate(c.spans):
        c.labels[a:b] = (c.x[a:b].double() @ c.w[w].double().T).argmax(1)
    c.forward()
    c.check_forward()
    some = 0
    for w, (a, b) in enumerate(c.spans):
        top = (c.x[a:b].double() @ c.w[w].double().T).topk(2, 1).values
        sure = top[:, 0] - top[:, 1] > 40.0
        some += int(sure.sum())
        assert (c.loss[a:b][sure] == 0).all() and (c.loss[a:b] >= 0).all()
    assert some > 10


@pytest.mark.parametrize("n_in", [9, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_single_class_costs_nothing(dtype, n_in):
    c = Case([40, 7], n_in, 1, dtype, spread=100.0)
    c.forward()
    assert (c.loss == 0).all()
    c.check_forward()
