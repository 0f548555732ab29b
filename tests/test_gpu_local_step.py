"""The operators of the local step together, as the example uses them: gradients of the whole chain against 64 bits,
and training that gets anywhere."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import local_step  # noqa: E402
import paper_1908_07782_b200 as combo  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_the_chain(dtype):
    counts, n_in, width, classes, groups = [40, 0, 75, 1], 24, 64, 10, 4
    w = local_step.Workers(counts, n_in, width, classes, groups, dtype)
    g = torch.Generator().manual_seed(0)
    w.params += (torch.randn(w.params.shape, generator=g) * 0.05).to(w.params)
    x, y = local_step.samples(counts, n_in, classes)
    w.sizes.clamp_(min=1.0)
    flat = w.params.to(dtype)
    w.grads.fill_(7.0)
    w.forward(x.to(dtype), flat)
    w.backward(x.to(dtype), y, flat)
    torch.cuda.synchronize()
    # the same in 64 bits by differentiation, from the values the kernels were given
    at = [0, 40, 40, 115, 116]
    # binary32: sums of at most 75 * 64 terms deep and two norms: 1e-4 of the largest gradient is far beyond it;
    # bfloat16: activations are rounded four times on the way, 2^-8 each, to gradients that are sums over samples
    tol = 1e-4 if dtype == torch.float32 else 6 * 2.0 ** -8
    for v in range(4):
        p = {k: w.view(flat, k)[v].double().cpu().requires_grad_() for k in w.places}
        xs, ys = x[at[v]:at[v + 1]].to(dtype).double().cpu(), y[at[v]:at[v + 1]].cpu()
        got = {k: w.view(w.grads, k)[v].double().cpu() for k in w.places}
        if len(ys) == 0:
            assert all((t == 0).all() for t in got.values())
            continue
        a = torch.nn.functional.silu(torch.nn.functional.group_norm(xs @ p["w1"].T, groups, p["gamma"], p["beta"], 1e-5))
        torch.nn.functional.cross_entropy(a @ p["w2"].T, ys).backward()
        for k, t in p.items():
            assert (got[k] - t.grad).abs().max() <= tol * t.grad.abs().max(), k
    # what lies between the layers is nobody's
    used = torch.zeros(w.P, dtype=torch.bool)
    for a, n, _ in w.places.values():
        used[a:a + n] = True
    assert (w.grads[:, ~used.to(w.grads.device)] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_lowers_the_loss(dtype):
    losses = local_step.main(["--rounds", "25", "--dtype", dtype, "--workers", "6"])
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0]


def test_one_round_is_the_clipped_step_and_the_aggregation():
    counts = [30, 50, 20, 44]
    w = local_step.Workers(counts, 16, 32, 4, 4)
    x, y = local_step.samples(counts, 16, 4)
    before = w.params.double().cpu().numpy()
    w.step(x, y, 0.25, 0.3, 0, segments=2, replicas=1)
    torch.cuda.synchronize()
    grads = w.grads.double().cpu().numpy()
    norms = np.sqrt((grads ** 2).sum(1))
    np.testing.assert_allclose(w.norm.cpu().numpy(), norms, rtol=1e-6)
    stepped = before - 0.25 * grads * np.minimum(1.0, 0.3 / (norms + 1e-6))[:, None]
    idx = torch.empty((4, 2, 1), dtype=torch.int32, device="cuda")
    combo.combo_select_peers(1, 0, 4, 2, 1, idx)
    idx, D = idx.cpu().numpy(), np.array(counts, dtype=np.float64)
    L = -(-w.P // 2)
    want = np.empty_like(stepped)
    for v in range(4):
        for s in range(2):
            k = idx[v, s, 0]
            c = slice(s * L, min((s + 1) * L, w.P))
            want[v, c] = (D[v] * stepped[v, c] + D[k] * stepped[k, c]) / (D[v] + D[k])
    # a handful of binary32 roundings of values up to max |stepped|
    assert np.abs(w.params.double().cpu().numpy() - want).max() <= 1e-6 * np.abs(stepped).max()
