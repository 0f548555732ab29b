"""Which of group norm's two ways sizes take, and both where several samples go to a CTA of the backward pass."""
import pytest
import torch

import paper_1908_07782_b200 as combo
from test_gpu_group_norm import ACTS, Case, check_backward, check_forward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
RESIDENT, STREAMED = combo.STEP_RESIDENT, combo.STEP_STREAMED


def ways(N, B, L, C, G, dtype):
    """The ways forward and backward go."""
    x = torch.randn(B, L, C, device=DEV).to(dtype)
    begin = torch.tensor([B * i // N for i in range(N + 1)], device=DEV)
    mean, rstd = torch.empty(B, G, device=DEV), torch.empty(B, G, device=DEV)
    scratch = torch.empty(combo.combo_group_norm_scratch_bytes(B, L, C, G), dtype=torch.uint8, device=DEV)
    p = torch.ones(N, C, device=DEV)
    y = torch.empty_like(x)
    combo.combo_group_norm(x, y, p, p, begin, G, 1e-5, 0, mean, rstd, scratch)
    first = combo.combo_last_step_path()
    combo.combo_group_norm_backward(y, x, torch.empty_like(x), p, p, begin, G, 0, mean, rstd, None, None, scratch)
    return first, combo.combo_last_step_path()


@pytest.mark.parametrize("N, B, L, C, G, dtype, taken", [
    (8, 1386, 1, 256, 8, torch.float32, (RESIDENT, STREAMED)),      # samples of one position behind a product
    (8, 1386, 1, 256, 8, torch.bfloat16, (RESIDENT, STREAMED)),
    (8, 8192, 1, 256, 8, torch.bfloat16, (RESIDENT, RESIDENT)),
    (8, 512, 4, 256, 8, torch.float32, (RESIDENT, STREAMED)),
    (8, 2048, 4, 256, 8, torch.float32, (RESIDENT, RESIDENT)),
    (8, 83, 49, 512, 32, torch.bfloat16, (RESIDENT, RESIDENT)),
    (8, 84, 49, 512, 32, torch.bfloat16, (RESIDENT, STREAMED)),     # x and dy are 8 MB and a little
    (8, 167, 49, 512, 32, torch.bfloat16, (STREAMED, STREAMED)),
    (8, 8, 49, 512, 32, torch.float32, (RESIDENT, RESIDENT)),
    (8, 1337, 49, 64, 8, torch.bfloat16, (RESIDENT, RESIDENT)),     # short samples, many workers to add their parameters' gradients
    (1, 1337, 49, 64, 8, torch.bfloat16, (RESIDENT, STREAMED)),
    (1, 160, 49, 256, 8, torch.bfloat16, (RESIDENT, STREAMED)),     # one worker's parameters, many samples
    (8, 160, 49, 256, 8, torch.bfloat16, (RESIDENT, RESIDENT)),
])
def test_ways(N, B, L, C, G, dtype, taken):
    assert ways(N, B, L, C, G, dtype) == taken


# workers that begin and end inside a CTA's samples, one that spans several, and some without any
MIX = [5, 0, 30, 2, 1, 12, 0, 0, 77, 3, 64]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("times, L, C, G, wide, taken", [
    (30, 1, 16, 2, 0, RESIDENT), (30, 1, 15, 3, 1, RESIDENT), (8, 4, 24, 4, 0, RESIDENT), (4, 8, 32, 8, 8, RESIDENT), (2, 24, 40, 5, 0, RESIDENT),
    (4, 1, 16, 2, 0, STREAMED), (4, 1, 15, 3, 1, STREAMED), (2, 4, 24, 4, 0, STREAMED), (1, 8, 32, 8, 8, STREAMED), (1, 31, 40, 5, 0, STREAMED),
])
def test_short_samples(dtype, times, L, C, G, wide, taken):
    for act in ACTS:
        c = Case(MIX * times, L, C, G, dtype, wide=wide, seed=act, pdtype=torch.bfloat16 if act == 1 else torch.float32)
        check_forward(c, act)
        check_backward(c, act)
        assert combo.combo_last_step_path() == taken
