"""Inputs and outputs of the local step's calls that are views beside each other in one wider array: they share no element, and
are not refused; those that do share one are."""
import ctypes

import pytest
import torch

import paper_1908_07782_b200 as combo

ALIAS = 2
DEV = "cuda:0"


@pytest.fixture()
def place():
    """A 16 KB host buffer, 256-byte aligned, for calls that are refused, or that find no GPU and read nothing."""
    if torch.cuda.is_available():
        pytest.skip("the calls that are not refused would run")
    buf = ctypes.create_string_buffer(16384 + 256)
    a = ctypes.addressof(buf)
    yield a + (-a) % 256
    del buf


def test_columns_that_share_elements_are_refused(place):
    lib = combo.load()
    need = combo.combo_group_norm_scratch_bytes(2, 4, 8, 2)
    scratch = place + 8192

    # floats, 8 channels at columns c and d of rows of 20
    def norm(c, d, xp=20, yp=20, B=2, L=4):
        return lib.combo_group_norm(place + 4 * c, xp, place + 4 * d, yp, 4, None, None, 4, 0, None, 1, B, L, 8, 2, 1e-5, 0, None, None,
                                    scratch, need, None)

    for c, d in ((0, 8), (8, 0), (0, 12), (12, 0), (2, 10), (4, 24 + 8), (20 + 8, 0)):
        assert norm(c, d) != ALIAS, (c, d)
    for c, d in ((0, 7), (7, 0), (0, 13), (13, 0), (0, 20), (4, 20), (12, 19), (3, 3 + 40)):
        assert norm(c, d) == ALIAS, (c, d)
    assert norm(5, 5) != ALIAS                                     # in place
    assert norm(0, 8, yp=24) == ALIAS and norm(0, 0, yp=24) == ALIAS
    assert norm(0, 8, yp=24, B=1, L=1) != ALIAS and norm(0, 0, yp=24, B=1, L=1) != ALIAS      # one row has no pitch
    assert norm(0, 4, B=1, L=1) == ALIAS

    # rows of 20 floats: 8 in, 6 out
    def linear(c, d, xp=20, yp=20, M=4, fn=lib.combo_grouped_linear, k=8, n=6):
        return fn(place + 4 * c, xp, place + 4096, 8, 48, place + 4 * d, yp, 4, 4, place + 8192, 2, M, k, n, None)

    for c, d in ((0, 8), (0, 14), (6, 0), (12, 6)):
        assert linear(c, d) != ALIAS, (c, d)
    for c, d in ((0, 7), (0, 15), (5, 0), (0, 20), (14, 0)):
        assert linear(c, d) == ALIAS, (c, d)
    back = lib.combo_grouped_linear_grad_input
    assert linear(0, 6, fn=back) != ALIAS and linear(0, 5, fn=back) == ALIAS and linear(0, 12, fn=back) != ALIAS
    assert linear(0, 8, yp=24) == ALIAS and linear(0, 1024) == ALIAS


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C, gap, L", [(32, 0, 40), (33, 1, 40), (64, 16, 30_000)])
def test_group_norm_beside_its_input(dtype, C, gap, L):
    g = torch.Generator(device=DEV).manual_seed(C)
    B, G = 3, 1 if C == 33 else 4
    wide = torch.randn(B, L, 3 * C + gap, generator=g, device=DEV).to(dtype)
    x, y, dx = wide[:, :, :C], wide[:, :, C:2 * C], wide[:, :, 2 * C + gap:]
    kept = wide.clone()
    apart, back = torch.empty(B, L, C, dtype=dtype, device=DEV), torch.empty(B, L, C, dtype=dtype, device=DEV)
    mean, rstd = torch.empty(B, G, device=DEV), torch.empty(B, G, device=DEV)
    scratch = torch.empty(combo.combo_group_norm_scratch_bytes(B, L, C, G), dtype=torch.uint8, device=DEV)
    dy = torch.randn(B, L, C, generator=g, device=DEV).to(dtype)

    def both(y, dx):
        combo.combo_group_norm(x, y, None, None, None, G, 1e-5, combo.ACT_RELU, mean, rstd, scratch)
        combo.combo_group_norm_backward(dy, x, dx, None, None, None, G, combo.ACT_RELU, mean, rstd, None, None, scratch)

    both(apart, back)
    both(y, dx)
    assert torch.equal(y, apart) and torch.equal(dx, back)
    assert torch.equal(x, kept[:, :, :C]) and torch.equal(wide[:, :, 2 * C:2 * C + gap], kept[:, :, 2 * C:2 * C + gap])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k, n, gap", [(64, 128, 0), (33, 20, 1), (512, 1024, 8)])
def test_products_beside_their_input(dtype, k, n, gap):
    g = torch.Generator(device=DEV).manual_seed(k)
    begin = torch.tensor([0, 70, 70, 101, 260], device=DEV)
    wide = torch.randn(260, k + gap + n, generator=g, device=DEV).to(dtype)
    w = torch.randn(4, n, k, generator=g, device=DEV).to(dtype)
    kept = wide.clone()
    x, y = wide[:, :k], wide[:, k + gap:]
    # an input of the same pitch elsewhere, so that both calls take the same kernel
    apart = torch.zeros_like(wide)[:, k + gap:]
    combo.combo_grouped_linear(x, w, apart, begin)
    combo.combo_grouped_linear(x, w, y, begin)
    assert torch.equal(y, apart) and torch.equal(wide[:, :k + gap], kept[:, :k + gap])
    wide.copy_(kept)
    dx = torch.zeros_like(wide)[:, :k]
    combo.combo_grouped_linear_grad_input(y, w, dx, begin)
    combo.combo_grouped_linear_grad_input(y, w, x, begin)
    assert torch.equal(x, dx) and torch.equal(wide[:, k:], kept[:, k:])
