"""combo_grad_norm, combo_grad_clip: norms over many tensors and clipping, against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
# Roundings, all terms of the sum being positive: a run of 16 squares is two chains of 8 FMAs and one addition (9 U of
# the sum, so 4.5 U of its root), the binary64 part is exact beside that, the root is rounded once.
NORM_TOL = 5.5 * U
# the coefficient: the norm's error, the addition of 1e-6, the division; then the product
OUT_TOL = NORM_TOL + 3 * U


class Lists:
    """N lists of tensors cut out of one buffer, `gap(i)` elements between them, and the table."""

    def __init__(self, sizes, dtype, seed=0, gap=lambda i: 0, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.N = sizes, len(sizes)
        flat, at, where = [], 8, []
        for w, mine in enumerate(sizes):
            for n in mine:
                at += gap(len(where))
                where.append((at, n))
                at += n
        self.buf = (torch.randn(at + 64, generator=g) * scale).to(dtype).to(DEV)
        self.where = where
        self.n = len(where)
        self.total = sum(n for _, n in where)
        e = self.buf.element_size()
        self.e = e
        self.offset = torch.tensor([a * e for a, _ in where], dtype=torch.int64)
        self.begin = torch.tensor(np.concatenate([[0], np.cumsum([n for _, n in where])]).astype(np.int64)).to(DEV)
        self.first = torch.tensor(np.concatenate([[0], np.cumsum([len(m) for m in sizes])]).astype(np.int32)).to(DEV)
        self.scratch = torch.full((combo.combo_grad_scratch_bytes(self.N) // 8,), float("nan"), dtype=torch.float64,
                                  device=DEV)

    def addresses(self, buf):
        return (self.offset + buf.data_ptr()).to(DEV)

    def check(self):
        return combo.combo_check_tensors(self.addresses(self.buf), self.begin, self.first, self.n, self.N, self.total,
                                         self.e)

    def clip(self, max_norm, out, out_shift=0):
        """Clips into `out` (a buffer like self.buf, or self.buf itself)."""
        norm = torch.full((self.N,), -1.0, device=DEV)
        coef = torch.full((self.N,), -1.0, device=DEV)
        dst = self.addresses(out) + out_shift * self.e
        combo.combo_grad_clip(self.addresses(self.buf), dst, self.begin, self.first, self.n, self.N, self.total, self.e,
                              max_norm, norm, coef, self.scratch)
        torch.cuda.synchronize()
        return norm, coef

    def norm(self, max_norm=1.0):
        norm = torch.full((self.N,), -1.0, device=DEV)
        coef = torch.full((self.N,), -1.0, device=DEV)
        combo.combo_grad_norm(self.addresses(self.buf), self.begin, self.first, self.n, self.N, self.total, self.e,
                              max_norm, norm, coef, self.scratch)
        torch.cuda.synchronize()
        return norm.cpu().numpy(), coef.cpu().numpy()

    def reference(self, max_norm):
        """norms, coefficients and clipped tensors in binary64."""
        x = self.buf.cpu().double().numpy()
        k, norms, coefs, outs = 0, [], [], []
        for mine in self.sizes:
            parts = []
            for _ in mine:
                a, n = self.where[k]
                parts.append(x[a:a + n])
                k += 1
            s = math.sqrt(sum(float(np.dot(p, p)) for p in parts))
            c = min(1.0, max_norm / (s + float(np.float32(1e-6))))
            norms.append(s)
            coefs.append(c)
            outs += [p * c for p in parts]
        return np.array(norms), np.array(coefs), outs


def half_ulp_bf16(v):
    return 0.5 * 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 7)


def check_outputs(t, out, outs, before, shift=0):
    got = out.cpu().double().numpy()
    touched = np.zeros(got.shape, bool)
    for (a, n), want in zip(t.where, outs):
        v = got[a + shift:a + shift + n]
        touched[a + shift:a + shift + n] = True
        tol = OUT_TOL * np.abs(want)
        if t.e == 2:
            tol = tol + half_ulp_bf16(np.abs(want) + tol)
        assert (np.abs(v - want) <= tol).all()
    assert (got[~touched] == before.cpu().double().numpy()[~touched]).all(), "written outside the tensors"


RAGGED = [
    [[1]],
    [[5], [1, 1, 1]],
    [[], [7], [], [3, 0, 4], []],
    [[4096]] * 3,
    [[1000, 1, 2, 3, 64, 64, 33333, 0, 17], [50001]],
    [[129] * 200, [2048] * 40, [1] * 90],
    [[1_000_003]],
    [[700_000, 5, 250_001]] * 5,
    [[3, 9]] * 700,                                     # far more workers than CTAs
    [[], []] + [[2_000_000, 77]] + [[]] * 3,
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", range(len(RAGGED)))
def test_clip_matches_formula(k, dtype):
    t = Lists(RAGGED[k], dtype, seed=k, gap=lambda i: (i * 7 + k) % 5)
    assert t.check() == 0
    max_norm = 0.5 * math.sqrt(max(1, t.total) / t.N)
    norms, coefs, outs = t.reference(max_norm)
    out = torch.full_like(t.buf, 3.0)
    before = out.clone()
    src = t.buf.clone()
    norm, coef = t.clip(max_norm, out)
    np.testing.assert_allclose(norm.cpu().numpy(), norms, rtol=NORM_TOL, atol=0)
    np.testing.assert_allclose(coef.cpu().numpy(), coefs, rtol=OUT_TOL, atol=0)
    check_outputs(t, out, outs, before)
    assert (t.buf == src).all()
    # norms alone, and the same in place
    n2, c2 = t.norm(max_norm)
    assert (n2 == norm.cpu().numpy()).all() and (c2 == coef.cpu().numpy()).all()
    t.clip(max_norm, t.buf)
    check_outputs(t, t.buf, outs, src)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_output_of_another_phase(dtype, shift):
    t = Lists([[10_001, 3, 7_000], [64, 5000]], dtype, seed=3, gap=lambda i: 8)
    _, _, outs = t.reference(2.0)
    out = torch.full_like(t.buf, 3.0)
    before = out.clone()
    t.clip(2.0, out, out_shift=shift)
    check_outputs(t, out, outs, before, shift=shift)


@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e-22, 1e15, 1e25, 1e37])
def test_norm_over_the_range_of_the_type(scale):
    # squares of these values leave binary32; the norms themselves do not
    t = Lists([[9_000], [40, 70], [0, 1]], torch.float32, seed=4, scale=scale / 100 if scale > 1 else scale)
    norms, coefs, _ = t.reference(1.0)
    norm, coef = t.norm()
    np.testing.assert_allclose(norm, norms, rtol=NORM_TOL, atol=2.0 ** -149)
    np.testing.assert_allclose(coef, coefs, rtol=OUT_TOL, atol=2.0 ** -149)


def test_zero_infinite_and_nan_gradients_stay_with_their_worker():
    t = Lists([[5000, 20], [300], [300], [300], [2500]], torch.float32, seed=5)
    where = dict(zip(range(6), t.where))
    t.buf[where[2][0] + 17] = float("inf")
    t.buf[where[3][0] + 299] = float("nan")
    t.buf[where[4][0]:where[4][0] + 300] = 0.0
    out = torch.full_like(t.buf, 3.0)
    norm, coef = t.clip(1.0, out)
    norm, coef = norm.cpu().numpy(), coef.cpu().numpy()
    assert np.isfinite(norm[[0, 3, 4]]).all() and norm[3] == 0.0 and coef[3] == 1.0
    assert norm[1] == np.inf and coef[1] == 0.0 and np.isnan(norm[2]) and np.isnan(coef[2])
    a, n = where[2]
    assert np.isnan(out[a + 17].item()) and (out[a:a + 17] == 0).all() and (out[a + 18:a + n] == 0).all()
    a, n = where[3]
    assert torch.isnan(out[a:a + n]).all()
    for k in (0, 1, 4, 5):
        a, n = where[k]
        assert torch.isfinite(out[a:a + n]).all()


def test_no_elements_at_all():
    for sizes in ([[], [], []], [[0], [0, 0]]):
        t = Lists(sizes, torch.float32)
        norm, coef = t.clip(2.0, t.buf)
        assert (norm == 0).all() and (coef == 1).all()
        norm, coef = t.norm(0.0)
        assert (norm == 0).all() and (coef == 0).all()


def test_limits_of_max_norm():
    t = Lists([[1000], [2000]], torch.float32, seed=6)
    src = t.buf.clone()
    out = torch.zeros_like(t.buf)
    _, coef = t.clip(float("inf"), out)
    assert (coef == 1).all()
    for a, n in t.where:
        assert (out[a:a + n] == src[a:a + n]).all()
    t.clip(0.0, out)
    for a, n in t.where:
        assert (out[a:a + n] == 0).all()


def test_same_result_every_time_and_on_another_stream():
    t = Lists([[300_000, 7, 123_457], [900_001]], torch.bfloat16, seed=7, gap=lambda i: i)
    a = t.norm()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = t.norm()
        out = torch.zeros_like(t.buf)
        t.clip(1.0, out)
    torch.cuda.synchronize()
    again = torch.zeros_like(t.buf)
    t.clip(1.0, again)
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
    assert torch.equal(out, again)


def test_rows_of_a_flat_array_beyond_32_bit_offsets():
    # two workers' rows, the second one beyond 2^32 bytes; small tensors at the far end
    P = 1_100_000_000
    x = torch.zeros(2, P, dtype=torch.bfloat16, device=DEV)
    x[0, :1000] = 1.0
    x[1, -501:] = 2.0
    begin = torch.tensor([0, P, 2 * P - 3, 2 * P], dtype=torch.int64, device=DEV)
    first = torch.tensor([0, 1, 3], dtype=torch.int32, device=DEV)
    at = (x.data_ptr() + torch.tensor([0, P, 2 * P - 3]) * 2).to(DEV)
    norm, coef = torch.zeros(2, device=DEV), torch.zeros(2, device=DEV)
    scratch = torch.empty(combo.combo_grad_scratch_bytes(2), dtype=torch.uint8, device=DEV)
    assert combo.combo_check_tensors(at, begin, first, 3, 2, 2 * P, 2) == 0
    combo.combo_grad_clip(at, at, begin, first, 3, 2, 2 * P, 2, 1.0, norm, coef, scratch)
    want = torch.tensor([1000.0, 4 * 501.0]).sqrt()
    np.testing.assert_allclose(norm.cpu().numpy(), want.numpy(), rtol=NORM_TOL)
    got = torch.stack([x[0, :1001], x[1, -1001:].flip(0)]).float().cpu()
    for w, (n, v) in enumerate(((1000, 1.0), (501, 2.0))):
        c = v / (float(want[w]) + 1e-6)
        assert (got[w, n:] == 0).all()
        assert (got[w, :n] - c).abs().max() <= half_ulp_bf16(np.float64(c)) + OUT_TOL * c


def test_refusals():
    t = Lists([[100], [50, 3]], torch.float32)
    norm = torch.zeros(2, device=DEV)
    a = t.addresses(t.buf)

    def refused(status=1, **kw):
        args = dict(tensors=a, out=a, begin=t.begin, first=t.first, n_tensors=3, N=2, total=153, elem_bytes=4, max_norm=1.0,
                    norm_out=norm, coef_out=None, scratch=t.scratch)
        args.update(kw)
        with pytest.raises(combo.ComboError) as e:
            combo.combo_grad_clip(**args)
        assert e.value.status == status
        args.pop("out")
        if "out" not in kw:
            with pytest.raises(combo.ComboError):
                combo.combo_grad_norm(**args)

    refused(elem_bytes=3)
    refused(N=0)
    refused(N=8193)
    refused(n_tensors=-1)
    refused(total=-1)
    refused(n_tensors=0)
    refused(max_norm=-1.0)
    refused(max_norm=float("nan"))
    refused(tensors=None)
    refused(out=None)
    refused(begin=None)
    refused(first=None)
    refused(scratch=None)
    refused(scratch=t.scratch[:8])
    assert combo.combo_grad_scratch_bytes(0) == 0
    # what the debug helper finds
    bad = t.begin.clone()
    bad[1] = 120
    assert combo.combo_check_tensors(a, bad, t.first, 3, 2, 153, 4) == 0        # still ascending
    bad[1] = 170
    assert combo.combo_check_tensors(a, bad, t.first, 3, 2, 153, 4) != 0
    assert combo.combo_check_tensors(a + 2, t.begin, t.first, 3, 2, 153, 4) == 3
    assert combo.combo_check_tensors(a, t.begin, t.first + 1, 3, 2, 153, 4) == 1 + 3 + 2
