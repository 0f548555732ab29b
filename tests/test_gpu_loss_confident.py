"""Rows whose label's class leads by far: their loss goes to zero and is never below, and so do their gradients, however large the
logits are."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1908_07782_b200 as combo  # noqa: E402
from loss_util import DEV, HALF, U, Case  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def confident(counts, n_in, n_out, dtype, lead, offset, **more):
    """Rows with one input of 1, so that logits are weights, which either type holds: the label's `offset`, the others' `lead` to
    `lead` + 24 below."""
    c = Case(counts, n_in, n_out, dtype, **more)
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


@pytest.mark.parametrize("offset,lead", [(20.0, 10.0), (250.0, 10.0), (250.0, 45.0), (-90.0, 45.0)])
@pytest.mark.parametrize("counts,n_in,n_out,path", [([3, 1, 20], 64, 10, combo.STEP_MULTIPLY_ADD), ([40, 130], 64, 700, combo.STEP_TENSOR),
                                                    ([40, 130], 600, 2000, combo.STEP_TENSOR), ([300, 200], 600, 1000, combo.STEP_TENSOR_PAIRS)])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "bf16-f32"])
def test_small_gradients_of_large_logits(types, counts, n_in, n_out, path, offset, lead):
    c = confident(counts, n_in, n_out, types[0], lead, offset, out=types[1], mean=False)
    lse = c.exact_lse()
    c.backward(lse)
    assert combo.combo_last_step_path() == path
    for w, (a, b) in enumerate(c.spans):
        x, wt, g, e = c.x[a:b].double(), c.w[w].double(), c.row_grad[a:b].double()[:, None], lse[a:b].double()[:, None]
        t = x @ wt.T - e
        hot = torch.zeros_like(t).scatter_(1, c.labels[a:b, None], 1.0)
        d = (torch.exp(t) - hot) * g
        # Logits are exact.  The difference to lse is rounded, and its product with log2(e); an exponential is off by 2^-22 of its
        # value; then come the difference to 1 and the factor.
        dd = g.abs() * (torch.exp(t) * (3 * t.abs() + 6) * U + 2.0 ** -126) + 2 * U * d.abs()
        n = b - a
        for got, want, tol, half in (
                (c.dx[a:b], d @ wt, (dd + HALF[types[0]] * d.abs()) @ wt.abs() + 2 * (n_out + 4) * U * (d.abs() @ wt.abs()), HALF[types[0]]),
                (c.dw[w], d.T @ x, (dd + (2.0 ** -16 if types[1] != types[0] else HALF[types[0]]) * d.abs()).T @ x.abs() +
                 2 * (n + 4) * U * (d.abs().T @ x.abs()), HALF[types[1]])):
            Case.near(got, want, tol, half, "gradients of worker %d" % w)
