"""Group norm streamed in two passes, as large batches take it: as many samples as fill the device (a chunk is a sample and a
thread walks many positions), and one sample cut into many chunks."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo
from test_gpu_group_norm import ACTS, DEV, EPS, U, Case, check_backward, check_forward, f64

pytestmark = pytest.mark.gpu
# workers without samples in front, between and behind
MANY = [0, 150, 0, 0, 1, 90, 61, 0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(300, 64, 8, 0), (301, 60, 4, 2)])        # the second: one element a load
def test_many_samples(dtype, shape):
    L, C, G, wide = shape
    for act in ACTS:
        c = Case(MANY, L, C, G, dtype, wide=wide, seed=act)
        check_forward(c, act)
        assert combo.combo_last_step_path() == combo.STEP_STREAMED
        check_backward(c, act)
        assert combo.combo_last_step_path() == combo.STEP_STREAMED


def test_a_large_mean():
    c = Case(MANY, 300, 64, 8, torch.float32, shift=3000.0, seed=2)
    check_forward(c, combo.ACT_NONE)
    assert combo.combo_last_step_path() == combo.STEP_STREAMED
    assert (c.rstd - 1.0).abs().max() < 0.2
    check_backward(c, combo.ACT_NONE)


def test_constant_input():
    c = Case(MANY, 300, 64, 8, torch.float32, seed=3)
    c.x.fill_(0.5)
    y = c.forward(combo.ACT_NONE)
    assert combo.combo_last_step_path() == combo.STEP_STREAMED
    assert (c.mean == 0.5).all() and (c.rstd - EPS ** -0.5).abs().max() <= 2e-7 * EPS ** -0.5
    assert torch.equal(y, c.beta.float()[torch.from_numpy(c.owner)][:, None, :].expand_as(y))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("counts, L", [(MANY, 300), ([1, 1], 40_000)])
def test_nan_and_infinity_stay_in_their_group(dtype, bad, counts, L):
    c = Case(counts, L, 64, 8, dtype, seed=4)
    clean = c.forward(combo.ACT_RELU).clone()
    dclean = c.backward(combo.ACT_RELU)[0].clone()
    for at in (0, 17, L - 1):
        keep = c.x[1, at, 20].clone()
        c.x[1, at, 20] = bad                        # group 2 of sample 1
        y = c.forward(combo.ACT_RELU)
        assert combo.combo_last_step_path() == combo.STEP_STREAMED
        m = torch.ones_like(y, dtype=torch.bool)
        m[1, :, 16:24] = False
        assert torch.equal(y[m], clean[m]) and torch.isnan(y[1, :, 16:24]).all()
        dx, dg, db = c.backward(combo.ACT_RELU)
        assert torch.equal(dx[m], dclean[m]) and torch.isnan(dx[1, :, 16:24]).all()
        w = int(c.owner[1])
        assert np.isnan(dg[w, 16:24]).all() and np.isfinite(np.delete(dg, w, 0)).all()
        assert np.isfinite(np.delete(dg[w], range(16, 24))).all()
        c.x[1, at, 20] = keep


def statistics(x, G, expect):
    """The call's statistics and those of 64 bits; its result is the formula's in binary32, from these statistics, bit for bit."""
    B, L, C = x.shape
    mean, rstd = torch.empty(B, G, device=DEV), torch.empty(B, G, device=DEV)
    scratch = torch.empty(combo.combo_group_norm_scratch_bytes(B, L, C, G), dtype=torch.uint8, device=DEV)
    y = torch.empty_like(x)
    combo.combo_group_norm(x, y, None, None, None, G, EPS, combo.ACT_NONE, mean, rstd, scratch)
    assert combo.combo_last_step_path() == expect
    xg = x.float().view(B, L, G, C // G)
    assert torch.equal(y, ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).view(B, L, C).to(x.dtype))
    var, m = torch.var_mean(xg.double(), dim=(1, 3), correction=0)
    return mean.double(), rstd.double(), m, 1.0 / torch.sqrt(var + EPS)


def check_statistics(x, G, run, lots):
    """`run`: positions that a thread adds one after another; `lots`: entries that are added one after another behind that,
    in the merge of a block and of the chunks.  M2 is a sum of positive terms, off by that many roundings of itself at most,
    twice as much where half of it is subtracted again (eight times in the first eight positions, which are few roundings),
    and rstd by half of that; 32 more for the trees, the division and the root."""
    mean, rstd, m, r = statistics(x, G, combo.STEP_STREAMED)
    assert ((rstd / r - 1).abs() <= (run + lots + 32) * U).all(), float((rstd / r - 1).abs().max() / U)
    # the mean: one rounding of a distance for every position, of sizes that fall as the pivot nears the mean
    size = x.float().abs().amax()
    assert ((mean - m).abs() <= 16 * U * size).all(), float((mean - m).abs().max() / (U * size))


@pytest.mark.parametrize("off", [0.0, 30.0, 100.0])
@pytest.mark.parametrize("B, L, C, G, dtype, run", [
    (300, 784, 64, 8, torch.float32, 98),
    (300, 784, 64, 1, torch.float32, 98),
    (230, 3136, 256, 32, torch.bfloat16, 784),
    (230, 3136, 512, 32, torch.float32, 3136),
    (230, 1301, 77, 7, torch.bfloat16, 1301),
])
def test_first_position_far_from_the_others(B, L, C, G, dtype, run, off):
    g = torch.Generator(device=DEV).manual_seed(7)
    x = torch.randn(B, L, C, generator=g, device=DEV)
    x[:, 0] += off
    check_statistics(x.to(dtype), G, run, 16)


@pytest.mark.parametrize("off", [0.0, 30.0, 100.0])
@pytest.mark.parametrize("B, L, C, G, run", [(1, 60_000, 64, 8, 17), (1, 400_000, 64, 32, 113), (4, 60_000, 64, 8, 68), (1, 50_001, 33, 3, 83)])
def test_first_chunk_far_from_the_others(B, L, C, G, run, off):
    g = torch.Generator(device=DEV).manual_seed(8)
    x = torch.randn(B, L, C, generator=g, device=DEV)
    x[:, :L // 400] += off
    check_statistics(x, G, run, 128)
