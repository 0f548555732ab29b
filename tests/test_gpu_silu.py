"""Group norm's SiLU and its slope far from zero, relative to their own size."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ULP = 2.0 ** -23
# exponential two units, quotient two, three roundings of half a unit
SILU_TOL = 5.5 * ULP
# the sigmoid s: exponential two units, quotient two, the sum under it and the product half a unit each; the bracket
# 1 + z (1 - s): where |z| >= 3 its larger term is at most 1.54 of it and off by 2.5 units (1 - s is 1 / (1 + e) there, or
# small), one rounding; two products; a rounding to spare
SLOPE_TOL = (5 + 1.54 * 2.5 + 0.5 + 1 + 0.5) * ULP
CENTRES = [0.0, -5.0, -10.0, -20.0, -30.0, -50.0, -80.0, -84.0, 5.0, 20.0, 60.0]


def inputs(centre, L, dtype=torch.float32):
    g = torch.Generator().manual_seed(int(centre) + 100)
    x = torch.randn(1, L, 512, generator=g).to(dtype).to(DEV)
    return x, torch.full((1, 512), 0.5, device=DEV), torch.full((1, 512), centre, device=DEV)


def forward(x, gamma, beta):
    L = x.shape[1]
    y, mean, rstd = torch.empty_like(x), torch.empty(1, 8, device=DEV), torch.empty(1, 8, device=DEV)
    scratch = torch.empty(combo.combo_group_norm_scratch_bytes(1, L, 512, 8), dtype=torch.uint8, device=DEV)
    combo.combo_group_norm(x, y, gamma, beta, None, 8, 1e-5, combo.ACT_SILU, mean, rstd, scratch)
    # z in the roundings that the call promises
    h = (x.float().view(1, L, 8, 64) - mean[:, None, :, None]) * rstd[:, None, :, None]
    z = h.reshape(1, L, 512) * gamma + beta
    return y, mean, rstd, scratch, z.double().cpu().numpy()


@pytest.mark.parametrize("L", [3, 40_000])                   # resident, streamed
@pytest.mark.parametrize("centre", CENTRES)
def test_silu(centre, L):
    y, _, _, _, z = forward(*inputs(centre, L))
    want = z / (1.0 + np.exp(-z))
    got = y.double().cpu().numpy()
    fine = np.abs(want) > 2.0 ** -120                        # far from where binary32's steps grow
    assert fine.all()
    assert (np.abs(got / want - 1.0) <= SILU_TOL).all(), float(np.abs(got / want - 1.0).max() / ULP)


@pytest.mark.parametrize("centre", [c for c in CENTRES if abs(c) >= 5])
def test_slope(centre):
    # one sample of one position: dbeta is dz itself
    x, gamma, beta = inputs(centre, 1)
    _, mean, rstd, scratch, z = forward(x, gamma, beta)
    dy, dx = torch.full_like(x, 1.25), torch.empty_like(x)
    dg, db = torch.empty(1, 512, device=DEV), torch.empty(1, 512, device=DEV)
    combo.combo_group_norm_backward(dy, x, dx, gamma, beta, None, 8, combo.ACT_SILU, mean, rstd, dg, db, scratch)
    s = 1.0 / (1.0 + np.exp(-z))
    one_less = 1.0 / (1.0 + np.exp(z))
    want = (1.25 * s * (1.0 + z * one_less)).reshape(-1)
    got = db.double().cpu().numpy().reshape(-1)
    assert (np.abs(got / want - 1.0) <= SLOPE_TOL).all(), float(np.abs(got / want - 1.0).max() / ULP)


@pytest.mark.parametrize("centre", CENTRES)
def test_silu_of_bfloat16(centre):
    y, _, _, _, z = forward(*inputs(centre, 300, torch.bfloat16))
    want = z / (1.0 + np.exp(-z))
    # rounded once to eight bits, and what is off before that
    tol = 1.01 * (2.0 ** -8 + (8 + 1.2 * np.abs(z)) * ULP)
    got = y.double().cpu().numpy()
    assert (np.abs(got / want - 1.0) <= tol).all(), float(np.abs(got / want - 1.0).max())
