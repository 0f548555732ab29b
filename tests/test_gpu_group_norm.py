"""combo_group_norm and combo_group_norm_backward against the formulas in 64 bits and against differences."""
import numpy as np
import pytest
import torch

import paper_1908_07782_b200 as combo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ACTS = [combo.ACT_NONE, combo.ACT_RELU, combo.ACT_SILU]
EPS = 1e-5


def half_ulp_bf16(v):
    return 0.5 * 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 7)


def f64(t):
    return t.detach().cpu().double().numpy()


class Case:
    """Inputs on the device, cut out of wider arrays with sentinels around the outputs."""

    def __init__(self, counts, L, C, G, dtype, pdtype=torch.float32, wide=0, seed=0, shift=0.0, affine=True, skew=0):
        g = torch.Generator().manual_seed(seed)
        self.counts, self.L, self.C, self.G, self.dtype = counts, L, C, G, dtype
        self.N, self.B = len(counts), sum(counts)
        self.begin = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)).to(DEV)
        self.owner = np.repeat(np.arange(self.N), counts)
        self.wide, self.skew = wide, skew

        def array(scale=1.0, offset=0.0):
            n = self.B * L * (C + wide)
            v = torch.randn(n + skew, generator=g) * scale + offset
            return v.to(dtype).to(DEV)[skew:].view(self.B, L, C + wide)[:, :, :C]

        self.x = array(1.0, shift)
        self.dy = array()
        flat = torch.randn(self.N, 2 * C + 7, generator=g) * 0.4
        flat[:, 1:C + 1] += 1.0
        self.flat = flat.to(pdtype).to(DEV)
        self.gamma = self.flat[:, 1:C + 1] if affine else None
        self.beta = self.flat[:, C + 4:2 * C + 4] if affine else None
        self.mean = torch.full((self.B, G), 7.0, device=DEV)
        self.rstd = torch.full((self.B, G), 7.0, device=DEV)

    def blank(self):
        self.buf = torch.full((self.B * self.L * (self.C + self.wide) + self.skew + 8,), 3.0, dtype=self.dtype, device=DEV)
        return self.buf[self.skew:self.skew + self.B * self.L * (self.C + self.wide)].view(
            self.B, self.L, self.C + self.wide)[:, :, :self.C]

    def untouched(self):
        m = torch.ones_like(self.buf, dtype=torch.bool)
        m[self.skew:self.skew + self.B * self.L * (self.C + self.wide)].view(
            self.B, self.L, self.C + self.wide)[:, :, :self.C] = False
        return bool((self.buf[m] == 3.0).all())

    def scratch(self):
        n = combo.combo_group_norm_scratch_bytes(self.B, self.L, self.C, self.G)
        return torch.full((n // 4,), float("nan"), device=DEV)

    def forward(self, act, y=None):
        y = self.blank() if y is None else y
        combo.combo_group_norm(self.x, y, self.gamma, self.beta, self.begin, self.G, EPS, act, self.mean, self.rstd,
                               self.scratch())
        torch.cuda.synchronize()
        return y

    def backward(self, act, dx=None, params=True):
        dx = self.blank() if dx is None else dx
        out = torch.full((self.N, 2 * self.C + 5), 3.0, device=DEV)
        dg, db = (out[:, 1:self.C + 1], out[:, self.C + 3:2 * self.C + 3]) if params else (None, None)
        combo.combo_group_norm_backward(self.dy, self.x, dx, self.gamma, self.beta, self.begin, self.G, act, self.mean,
                                        self.rstd, dg, db, self.scratch())
        torch.cuda.synchronize()
        if params:
            out[:, 1:self.C + 1], kept = -1.0, out[:, 1:self.C + 1].clone()
            out[:, self.C + 3:2 * self.C + 3], kept2 = -1.0, out[:, self.C + 3:2 * self.C + 3].clone()
            assert ((out == -1.0) | (out == 3.0)).all(), "written between the parameters"
            return dx, f64(kept), f64(kept2)
        return dx

    # ------------------------------------------------------------ 64 bits
    def per_sample(self):
        ga = np.ones((self.N, self.C)) if self.gamma is None else f64(self.gamma)
        be = np.zeros((self.N, self.C)) if self.beta is None else f64(self.beta)
        return ga[self.owner][:, None, :], be[self.owner][:, None, :]

    def grouped(self, v):
        return v.reshape(self.B, self.L, self.G, self.C // self.G)

    def spread(self, v):
        """[B, G] -> [B, 1, C]."""
        return np.repeat(v, self.C // self.G, axis=1)[:, None, :]


def act64(z, act):
    with np.errstate(over="ignore"):
        return z if act == 0 else np.maximum(z, 0.0) if act == 1 else z / (1.0 + np.exp(-z))


def depth(c):
    """Additions one after another behind any sum: a thread's positions (at most 256 in these cases) and the merge of
    its block's entries, 64 at most in a lane, then trees."""
    return min(c.L, 256) + 80


def check_forward(c, act):
    y = c.forward(act)
    if c.B == 0:
        return
    x = f64(c.x)
    xg = c.grouped(x)
    mean, var = xg.mean(axis=(1, 3)), xg.var(axis=(1, 3))
    rstd = 1.0 / np.sqrt(var + EPS)
    big = np.abs(xg).max(axis=(1, 3))
    D = depth(c)
    # mean: D additions of values up to `big`; the deviations inherit it, and their squares are added D deep
    dm = (D + 4) * U * big
    dr = rstd * ((D + 8) * U + (dm * rstd) ** 2 + dm * rstd * (D + 8) * U)
    assert (np.abs(f64(c.mean) - mean) <= dm).all()
    assert (np.abs(f64(c.rstd) - rstd) <= dr).all()
    ga, be = c.per_sample()
    h = (x - c.spread(mean)) * c.spread(rstd)
    dh = c.spread(dm * rstd) + np.abs(h) * (c.spread(dr / rstd) + 4 * U)
    z = h * ga + be
    dz = np.abs(ga) * dh + 2 * U * (np.abs(h * ga) + np.abs(be)) + U * np.abs(z)
    want = act64(z, act)
    tol = 1.1 * dz + U * np.abs(want)
    if act == combo.ACT_SILU:      # exponential, division: some units in the last place, growing with the argument
        tol = tol + (np.abs(z) + 1.0) * 2.0 ** -20
    if c.dtype == torch.bfloat16:
        tol = tol + half_ulp_bf16(np.abs(want) + tol)
    got = f64(y)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
    assert c.untouched(), "written outside the output"


def check_backward(c, act):
    dx, dg, db = c.backward(act)
    D = depth(c)
    if c.B:
        x, dy = f64(c.x), f64(c.dy)
        ga, be = c.per_sample()
        # h and z in the roundings that the call promises decide what ReLU clipped
        f = np.float32
        x32, m32, r32 = x.astype(f), c.spread(f64(c.mean)).astype(f), c.spread(f64(c.rstd)).astype(f)
        z32 = ((x32 - m32) * r32 * ga.astype(f)).astype(f) + be.astype(f)
        h = (x - c.spread(f64(c.mean))) * c.spread(f64(c.rstd))
        z = h * ga + be
        dh = 3 * U * np.abs(h)
        s = 1.0 / (1.0 + np.exp(-z))
        slope = np.ones_like(z) if act == 0 else (z32 > 0).astype(float) if act == 1 else s * (1 + z * (1 - s))
        dz = dy * slope
        ddz = np.zeros_like(dz)
        if act == combo.ACT_SILU:
            ddz = np.abs(dy) * (0.5 * (np.abs(ga) * dh + 3 * U * (np.abs(h * ga) + np.abs(be))) + (np.abs(z) + 2) * 2.0 ** -20)
        t, rs = dz * ga, c.spread(f64(c.rstd))
        dt = np.abs(ga) * ddz + U * np.abs(t)

        def mean(v):
            return c.spread(c.grouped(v).mean(axis=(1, 3)))

        m1, m2 = mean(t), mean(t * h)
        dm1 = mean(dt) + (D + 4) * U * mean(np.abs(t))
        dm2 = mean(dt * np.abs(h)) + (D + 8) * U * mean(np.abs(t * h))
        want = rs * (t - m1 - h * m2)
        tol = np.abs(rs) * (dt + dm1 + np.abs(h) * dm2 + dh * np.abs(m2) + 4 * U * (np.abs(t) + np.abs(m1) + np.abs(h * m2)))
        if c.dtype == torch.bfloat16:
            tol = tol + half_ulp_bf16(np.abs(want) + tol)
        got = f64(dx)
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
        assert c.untouched(), "written outside the output"
    for w in range(c.N):
        mine = c.owner == w
        if not mine.any():
            assert (dg[w] == 0).all() and (db[w] == 0).all()
            continue
        k = int(mine.sum())
        for got, terms, err in ((dg[w], (dz * h)[mine], (ddz * np.abs(h) + np.abs(dz) * dh)[mine]), (db[w], dz[mine], ddz[mine])):
            want = terms.sum(axis=(0, 1))
            tol = err.sum(axis=(0, 1)) + (D + k + 8) * U * np.abs(terms).sum(axis=(0, 1))
            assert (np.abs(got - want) <= tol).all()


SHAPES = [
    # counts, L, C, groups, elements between positions beside C, elements before the first
    ([1], 2, 1, 1, 0, 0),
    ([2, 0, 1], 1, 6, 2, 0, 0),
    ([3], 5, 6, 2, 3, 1),
    ([1, 2], 49, 512, 32, 0, 0),
    ([0, 3, 0, 2, 0], 33, 64, 32, 0, 0),           # 2 channels a group: a 16-byte vector spans groups
    ([2, 1], 100, 128, 32, 8, 8),
    ([1, 1], 784, 96, 3, 0, 0),
    ([1], 3136, 256, 32, 0, 0),                    # a long sample
    ([1, 1], 3137, 40, 4, 0, 0),                   # the same, ragged
    ([1], 997, 3, 3, 0, 0),                        # one channel a group, odd
    ([2], 7, 77, 7, 5, 3),
    ([1], 20_001, 64, 1, 0, 0),                    # too long for shared memory: streamed
    ([1], 9_001, 61, 1, 0, 0),
    ([2, 1], 3, 4096, 1, 0, 0),                    # more vectors than threads
    ([1], 2, 2600, 2, 1, 0),
    ([5, 0, 30, 2, 1, 12], 1, 48, 4, 0, 0),        # short samples: several to a CTA, workers changing inside
    ([1] * 40 + [0] * 5 + [7], 4, 16, 2, 0, 0),
    ([1] * 300, 2, 8, 1, 0, 0),
    ([3, 0, 2], 1500, 512, 32, 0, 0),              # streamed for its size, chunks of unequal length
    ([2, 1], 1300, 1026, 18, 2, 0),                # the same, 57 channels a group, no whole vectors
    ([2], 700, 2304, 9, 8, 8),                     # more vectors than threads in a block
    ([1, 1], 3001, 128, 32, 0, 0),                 # streamed, 4 channels a group
    ([2], 7000, 64, 32, 8, 0),                     # streamed, 2 channels a group
    ([1, 0, 2], 5000, 24, 8, 0, 0),                # streamed, 3 channels a group
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", range(len(SHAPES)))
def test_forward_and_backward_match_formulas(k, dtype):
    counts, L, C, G, wide, skew = SHAPES[k]
    for act in ACTS:
        c = Case(counts, L, C, G, dtype, wide=wide, skew=skew, seed=10 * k + act,
                 pdtype=torch.bfloat16 if (k + act) % 3 == 0 else torch.float32)
        check_forward(c, act)
        check_backward(c, act)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_parameters_and_one_worker_without_a_table(dtype):
    c = Case([3], 50, 32, 4, dtype, affine=False, seed=1)
    c.begin = None
    check_forward(c, combo.ACT_SILU)
    check_backward(c, combo.ACT_SILU)
    # statistics and parameter gradients not wanted
    y = c.forward(combo.ACT_RELU).clone()
    c2 = c.blank()
    combo.combo_group_norm(c.x, c2, None, None, None, 4, EPS, combo.ACT_RELU, None, None, c.scratch())
    assert torch.equal(y, c2)
    dx = c.backward(combo.ACT_RELU)[0].clone()
    assert torch.equal(dx, c.backward(combo.ACT_RELU, params=False))


def test_a_large_mean_costs_nothing():
    # deviations of size 1 on a mean of 3000: squares of the values would leave binary32 with nothing
    c = Case([2, 1], 500, 64, 8, torch.float32, shift=3000.0, seed=2)
    check_forward(c, combo.ACT_NONE)
    assert (c.rstd - 1.0).abs().max() < 0.2
    check_backward(c, combo.ACT_NONE)


def test_constant_input():
    c = Case([2], 60, 32, 4, torch.float32, seed=3)
    c.x.fill_(0.5)
    y = c.forward(combo.ACT_NONE)
    assert (c.mean == 0.5).all() and (c.rstd - EPS ** -0.5).abs().max() <= 2e-7 * EPS ** -0.5
    assert torch.equal(y, c.beta.float().expand(2, 60, 32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nan_and_infinity_stay_in_their_group(dtype, bad):
    c = Case([2, 1], 300, 64, 8, dtype, seed=4)
    clean = c.forward(combo.ACT_RELU).clone()
    dclean = c.backward(combo.ACT_RELU)[0].clone()
    c.x[1, 17, 20] = bad                            # group 2 of sample 1
    y = c.forward(combo.ACT_RELU)
    m = torch.ones_like(y, dtype=torch.bool)
    m[1, :, 16:24] = False
    assert torch.equal(y[m], clean[m]) and torch.isnan(y[1, :, 16:24]).all()
    dx, dg, db = c.backward(combo.ACT_RELU)
    assert torch.equal(dx[m], dclean[m]) and torch.isnan(dx[1, :, 16:24]).all()
    assert np.isnan(dg[0, 16:24]).all() and np.isfinite(dg[1]).all() and np.isfinite(np.delete(dg[0], range(16, 24))).all()


def test_gradients_where_relu_clipped_are_dropped():
    c = Case([1], 64, 32, 4, torch.float32, seed=5)
    y = c.forward(combo.ACT_RELU)
    want = c.backward(combo.ACT_RELU)[0].clone()
    c.dy[y == 0] = float("inf")
    assert torch.equal(want, c.backward(combo.ACT_RELU)[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(3136, 128, 8), (40, 24, 3), (20_001, 64, 1)])
def test_in_place_and_another_stream_and_every_time_the_same(dtype, shape):
    L, C, G = shape
    c = Case([1, 1], L, C, G, dtype, seed=6)
    y = c.forward(combo.ACT_SILU).clone()
    dx, dg, db = c.backward(combo.ACT_SILU)
    dx = dx.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = c.backward(combo.ACT_SILU)
    assert torch.equal(again[0], dx) and (again[1] == dg).all() and (again[2] == db).all()
    x, dy = c.x.clone(), c.dy.clone()
    c.backward(combo.ACT_SILU, dx=c.dy)
    assert torch.equal(c.dy, dx)
    c.dy = dy
    c.backward(combo.ACT_SILU, dx=c.x)
    assert torch.equal(c.x, dx)
    c.x = x
    c.forward(combo.ACT_SILU, y=c.x)
    assert torch.equal(c.x, y)


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    c = Case([2, 1], 20, 24, 3, torch.float32, seed=7)
    c.forward(act)
    dx, dg, db = c.backward(act)
    g = np.random.RandomState(0)
    x, dy = f64(c.x), f64(c.dy)
    ga, be = f64(c.gamma), f64(c.beta)

    def loss(x, ga, be):
        xg = c.grouped(x)
        h = (xg - xg.mean(axis=(1, 3), keepdims=True)) / np.sqrt(xg.var(axis=(1, 3), keepdims=True) + EPS)
        return float((dy * act64(h.reshape(x.shape) * ga[c.owner][:, None] + be[c.owner][:, None], act)).sum())

    for which, grad in ((0, f64(dx)), (1, dg), (2, db)):
        at = [x, ga, be]
        v = g.randn(*at[which].shape)
        # small enough that ReLU clips the same values on both sides but for a few, whose share is below e
        e = 1e-6
        plus, minus = list(at), list(at)
        plus[which] = at[which] + e * v
        minus[which] = at[which] - e * v
        diff = (loss(*plus) - loss(*minus)) / (2 * e)
        got = float((grad * v).sum())
        # differences: e^2 of the third derivative and rounding of the loss, 1e-16 * |loss| / e; the gradient: binary32
        assert abs(diff - got) <= 1e-4 * max(1.0, float(np.abs(grad * v).sum())) * 0.1


def test_many_positions_in_one_worker_at_large_offsets():
    # samples beyond 2^32 bytes of the array
    L, C = 1 << 20, 64
    x = torch.zeros(40, L, C, dtype=torch.bfloat16, device=DEV)
    x[39, :, 1::2] = 2.0
    mean, rstd = torch.empty(40, 8, device=DEV), torch.empty(40, 8, device=DEV)
    scratch = torch.empty(combo.combo_group_norm_scratch_bytes(40, L, C, 8), dtype=torch.uint8, device=DEV)
    combo.combo_group_norm(x, x, None, None, None, 8, EPS, combo.ACT_NONE, mean, rstd, scratch)
    assert (mean[:39] == 0).all() and (mean[39] - 1.0).abs().max() <= 1e-6
    assert (x[:39] == 0).all()
    assert (x[39, :, 1::2] == 1.0).all() and (x[39, :, ::2] == -1.0).all()


def test_refusals():
    c = Case([1, 2], 10, 24, 3, torch.float32)
    y = c.blank()

    def refused(status=1, **kw):
        args = dict(x=c.x, y=y, gamma=c.gamma, beta=c.beta, begin=c.begin, groups=3, eps=EPS, act=0, mean=c.mean, rstd=c.rstd,
                    scratch=c.scratch())
        args.update(kw)
        with pytest.raises(combo.ComboError) as e:
            combo.combo_group_norm(**args)
        assert e.value.status == status

    refused(groups=5, mean=None, rstd=None)
    refused(groups=0, mean=None, rstd=None)
    refused(act=3)
    refused(eps=-1.0)
    refused(eps=float("nan"))
    refused(beta=None)
    shifted = torch.zeros(3 * 10 * 24 + 24, device=DEV)
    refused(status=2, x=shifted[:720].view(3, 10, 24), y=shifted[24:].view(3, 10, 24))
    with pytest.raises(ValueError):
        combo.combo_group_norm(c.x.transpose(1, 2), y, c.gamma, c.beta, c.begin, 3, EPS, 0, None, None, c.scratch())
    with pytest.raises(ValueError):
        combo.combo_group_norm(c.x, y, c.gamma.double(), c.beta.double(), c.begin, 3, EPS, 0, None, None, c.scratch())
    with pytest.raises(ValueError):
        combo.combo_group_norm(c.x, y, c.gamma, c.beta, c.begin[:-1], 3, EPS, 0, None, None, c.scratch())
    c.forward(0)
    s = torch.empty(combo.combo_group_norm_scratch_bytes(3, 10, 24, 3) - 8, dtype=torch.uint8, device=DEV)
    with pytest.raises(combo.ComboError):
        combo.combo_group_norm_backward(c.dy, c.x, y, c.gamma, c.beta, c.begin, 3, 0, c.mean, c.rstd, None, None, s)
    with pytest.raises(combo.ComboError):
        combo.combo_group_norm_backward(c.dy, c.x, y, c.gamma, c.beta, c.begin, 3, 0, c.mean, c.rstd, None, None, None)
    wide = Case([1], 1, 4097, 1, torch.float32)
    with pytest.raises(combo.ComboError):
        wide.forward(0)
    assert combo.combo_group_norm_scratch_bytes(1, 0, 4, 1) == 0
    refused(scratch=None)
    refused(scratch=s)
