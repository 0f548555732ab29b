"""The grouped cross entropy where the classes are taken in several pieces, and at the largest numbers of classes and inputs."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1908_07782_b200 as combo  # noqa: E402
from loss_util import Case  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,out,counts,n_in,n_out", [(BF16, F32, [2100, 2000], 64, 66000), (F32, F32, [1200, 900], 40, 90000),
                                                         (BF16, BF16, [3000, 70], 72, 180001)])
def test_gradients_in_pieces(dtype, out, counts, n_in, n_out):
    # d alone is more than a piece's gigabyte
    planes = 3 if dtype == F32 else 2 if out == F32 else 1
    assert sum(counts) * n_out * 2 * planes > 1 << 30
    c = Case(counts, n_in, n_out, dtype, out)
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


def test_loss_in_pieces():
    """Float weights whose planes are more than a gigabyte."""
    c = Case([1] * 64, 1000, 4500, F32)
    assert 64 * 4500 * 1024 * 4 > 1 << 30
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,n_in,n_out", [([3], 16, 1 << 20), ([2, 1], 1 << 20, 8)])
def test_the_most_classes_and_inputs(counts, n_in, n_out, dtype):
    c = Case(counts, n_in, n_out, dtype)
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)
    combo.combo_device_status()


def test_many_rows_of_few_labels():
    c = Case([30000, 0, 9000], 40, 70, BF16, F32, keep=0.02, mean=False)
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_most_workers(dtype):
    c = Case([k % 3 == 0 for k in range(8192)], 16, 300, dtype)
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


def test_loss_in_pieces_off_16_bytes():
    """bfloat16 weights whose copy is more than a gigabyte."""
    assert 8 * 70001 * 1024 * 2 > 1 << 30
    c = Case([3, 1, 0, 2, 1, 5, 1, 1], 1000, 70001, BF16, xp=3, wp=1, skew=1)
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("dtype,out,counts,n_in,n_out", [(BF16, F32, [2100, 2000], 61, 66000), (F32, F32, [1200, 900], 39, 90000),
                                                         (BF16, BF16, [3000, 70], 77, 180001)])
def test_gradients_in_pieces_off_16_bytes(dtype, out, counts, n_in, n_out):
    planes = 3 if dtype == F32 else 2 if out == F32 else 1
    assert sum(counts) * n_out * 2 * planes > 1 << 30
    c = Case(counts, n_in, n_out, dtype, out, xp=3, wp=1, skew=1, mean=False)
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


def test_pieces_sum_alike():
    """Classes of equal weights, one in every 256, lie at the same places of the tiles of every piece: wherever no row has them as its
    label their gradients are equal to the last bit."""
    counts, n_in, n_out = [2100, 2000], 520, 256 * 258
    assert sum(counts) * n_out * 2 * 2 > 1 << 30               # d alone is more than a piece
    c = Case(counts, n_in, n_out, BF16, F32)
    c.w.copy_(c.w[:, :256].repeat(1, n_out // 256, 1))
    c.labels %= 256
    c.forward()
    c.backward(c.lse)
    dw = c.dw.view(2, n_out // 256, 256, n_in)
    assert torch.equal(dw[:, 1:], dw[:, 1:2].expand(-1, n_out // 256 - 1, -1, -1))


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "bf16-f32"])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("counts,n_in,n_out", [([129, 65, 0, 257], 200, 1500), ([40, 3], 136, 2057), ([300, 200], 776, 1301), ([700] * 3, 520, 20)])
def test_the_least_scratch(counts, n_in, n_out, odd, types):
    """Pieces of one tile of classes; the same values from any amount of scratch, rows' gradients up to the order of their sums."""
    c = Case(counts, n_in, n_out, types[0], types[1], keep=0.8, mean=False, xp=3 * odd, wp=odd, skew=odd)
    size = {F32: 4, BF16: 2}
    least = [combo.combo_grouped_cross_entropy_least_scratch_bytes(c.N, c.M, n_in, n_out, size[types[0]], g) for g in (0, size[types[1]])]
    lse = c.exact_lse()
    want = []
    for more in (0, 1 << 20, 1 << 30):
        # nothing behind what was given is touched
        f, b = (torch.full((n + more + 4096,), 0xff, dtype=torch.uint8, device="cuda:0") for n in least)
        c.forward(f[:least[0] + more])
        c.check_forward()
        c.backward(lse, b[:least[1] + more])
        c.check_backward(lse)
        assert (f[least[0] + more:] == 0xff).all() and (b[least[1] + more:] == 0xff).all()
        want.append([t.clone() for t in (c.loss, c.lse, c.dw)])
    for got in want[1:]:
        assert all(torch.equal(a, k) for a, k in zip(got, want[0]))


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "bf16-f32"])
def test_many_workers_of_few_classes(types):
    """Planes of the classes there are: 20 and not a tile's 128."""
    c = Case([k % 5 for k in range(1200)], 136, 20, types[0], types[1], keep=0.8, xp=3, wp=1, skew=1)
    c.forward()
    assert combo.combo_last_step_path() == combo.STEP_TENSOR
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)


def test_the_most_rows():
    """Scratch of more than a gigabyte for one tile of classes."""
    c = Case([1 << 21, 0, (1 << 21) - 7, 2], 24, 70, BF16, F32, keep=0.6, mean=False, lead=2, behind=3)
    assert c.M == 1 << 22
    c.forward()
    c.check_forward()
    lse = c.exact_lse()
    c.backward(lse)
    c.check_backward(lse)
    combo.combo_device_status()
