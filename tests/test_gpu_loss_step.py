"""The local step's whole chain with dropout and the grouped cross entropy, as the example runs it: gradients against 64 bits,
the same bits from a captured graph, and which kernels the loss takes."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import local_step  # noqa: E402
import paper_1908_07782_b200 as combo  # noqa: E402
from loss_util import Case  # noqa: E402

pytestmark = pytest.mark.gpu


def mask(w, rnd):
    """What dropout keeps, scaled, of every activation."""
    t = torch.ones(w.M, w.width, dtype=torch.float32, device=w.device)
    combo.combo_dropout(t, None, t, w.begin, w.dropout, w.seed, rnd)
    return t


@pytest.mark.parametrize("classes", [10, 700])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_with_dropout(dtype, classes):
    counts, n_in, width, groups, rnd = [40, 0, 75, 1], 24, 64, 4, 3
    w = local_step.Workers(counts, n_in, width, classes, groups, dtype, dropout=0.2)
    g = torch.Generator().manual_seed(0)
    w.params += (torch.randn(w.params.shape, generator=g) * 0.05).to(w.params)
    x, y = local_step.samples(counts, n_in, classes)
    y[5] = y[50] = -1                                    # samples without a label
    flat = w.params.to(dtype)
    w.forward(x.to(dtype), flat, rnd)
    loss = w.backward(x.to(dtype), y, flat, rnd)
    kept = mask(w, rnd).double().cpu()
    assert 0.1 < float((kept == 0).double().mean()) < 0.3
    at = [0, 40, 40, 115, 116]
    # as the chain without dropout: 1e-4 of the largest gradient; bfloat16 activations are rounded six times on the way, 2^-8
    # each (the branch's scale among them)
    tol = 1e-4 if dtype == torch.float32 else 8 * 2.0 ** -8
    for v in range(4):
        p = {k: w.view(flat, k)[v].double().cpu().requires_grad_() for k in w.places}
        xs, ys = x[at[v]:at[v + 1]].to(dtype).double().cpu(), y[at[v]:at[v + 1]].cpu()
        got = {k: w.view(w.grads, k)[v].double().cpu() for k in w.places}
        if len(ys) == 0:
            assert all((t == 0).all() for t in got.values())
            continue
        a = torch.nn.functional.silu(torch.nn.functional.group_norm(xs @ p["w1"].T, groups, p["gamma"], p["beta"], 1e-5))
        z = (a * kept[at[v]:at[v + 1]]) @ p["w2"].T
        want = torch.nn.functional.cross_entropy(z, ys, ignore_index=-1, reduction="none")
        # logits of a few units from activations rounded twice
        assert (loss[at[v]:at[v + 1]].double().cpu() - want).abs().max() <= (1e-4 if dtype == torch.float32 else 0.1)
        (want.sum() / (ys >= 0).sum()).backward()
        for k, t in p.items():
            assert (got[k] - t.grad).abs().max() <= tol * t.grad.abs().max(), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_while_an_eager_pass_lives(dtype):
    """Forward and backward captured into a graph between eager passes of the same buffers."""
    counts = [130, 60, 0, 33]
    w = local_step.Workers(counts, 32, 128, 500, 4, dtype, dropout=0.1)
    x, y = local_step.samples(counts, 32, 500)
    flat, xt = w.params.to(dtype), x.to(dtype)

    def both():
        w.forward(xt, flat, 1)
        w.backward(xt, y, flat, 1)

    both()
    torch.cuda.synchronize()
    want = [w.loss.clone(), w.grads.clone()]
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both()
    both()
    for _ in range(2):
        w.loss.zero_()
        w.grads.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w.loss, want[0]) and torch.equal(w.grads, want[1])


def test_training_with_dropout_runs():
    assert len(local_step.main(["--rounds", "3", "--dropout", "0.2", "--dtype", "bf16"])) == 3


def test_which_kernels_a_loss_takes():
    for counts, n_in, n_out, path in (([40, 9], 64, 20, combo.STEP_MULTIPLY_ADD), ([40, 9], 256, 3000, combo.STEP_TENSOR),
                                      ([300, 200], 520, 3000, combo.STEP_TENSOR_PAIRS), ([1500, 900], 64, 20, combo.STEP_TENSOR)):
        for dtype in (torch.float32, torch.bfloat16):
            c = Case(counts, n_in, n_out, dtype)
            c.forward()
            assert combo.combo_last_step_path() == path
            c.backward(c.lse)
            assert combo.combo_last_step_path() == path
