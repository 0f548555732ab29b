"""Inputs, definitions in 64 bits and error bounds for the tests of the grouped cross entropy."""
import numpy as np
import torch

import paper_1908_07782_b200 as combo

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


def rows_array(M, width, pitch, dtype, g, skew=0):
    """[M, width] with `pitch` elements between rows, `skew` before the first; NaN everywhere else."""
    buf = torch.full((skew + M * pitch + 16,), float("nan"), dtype=dtype, device=DEV)
    t = buf[skew:skew + M * pitch].view(M, pitch)[:, :width]
    t.copy_(torch.randn(M, width, generator=g))
    return buf, t


def weight_array(N, n_out, n_in, pitch, gap, dtype, g, skew=0, scale=1.0):
    stride = n_out * pitch + gap
    buf = torch.full((skew + N * stride + 16,), float("nan"), dtype=dtype, device=DEV)
    t = buf.as_strided((N, n_out, n_in), (stride, pitch, 1), skew)
    t.copy_(torch.randn(N, n_out, n_in, generator=g) * scale)
    return buf, t


class Case:
    """One set of inputs; `keep` of the rows have a label."""

    def __init__(self, counts, n_in, n_out, dtype, out=None, keep=1.0, mean=True, xp=0, wp=0, gap=0, skew=0, lead=0, behind=0, seed=0,
                 spread=1.5):
        g = torch.Generator().manual_seed(seed)
        self.counts, self.N, self.K, self.V, self.dtype, self.out = counts, len(counts), n_in, n_out, dtype, out or dtype
        self.M = lead + sum(counts) + behind
        at = lead + np.concatenate([[0], np.cumsum(counts)])
        self.spans = list(zip(at[:-1].tolist(), at[1:].tolist()))
        self.begin = torch.tensor(at.astype(np.int64)).to(DEV)
        _, self.x = rows_array(self.M, n_in, n_in + xp, dtype, g, skew)
        _, self.w = weight_array(self.N, n_out, n_in, n_in + wp, gap, dtype, g, skew, spread / n_in ** 0.5)
        labels = torch.randint(0, n_out, (self.M,), generator=g)
        none = torch.rand(self.M, generator=g) >= keep
        labels[none] = torch.tensor([-100, -1, n_out, 1 << 40])[torch.randint(0, 4, (int(none.sum()),), generator=g)]
        self.labels = labels.to(DEV)
        self.has = (self.labels >= 0) & (self.labels < n_out)
        # what has no label may hold anything
        self.x[~self.has] = float("nan")
        self.loss, self.lse = (torch.full((self.M,), 7.0, device=DEV) for _ in range(2))
        self.row_grad = None if mean else torch.rand(self.M, generator=g).to(DEV) - 0.25
        self.dx_buf, self.dx = rows_array(self.M, n_in, n_in + xp, dtype, g, skew)
        self.dw_buf, self.dw = weight_array(self.N, n_out, n_in, n_in + wp, gap, self.out, g, skew)
        self.inside = torch.zeros(self.M, dtype=torch.bool, device=DEV)
        self.inside[at[0]:at[-1]] = True

    def scratch(self, back):
        size = {torch.float32: 4, torch.bfloat16: 2}
        n = combo.combo_grouped_cross_entropy_scratch_bytes(self.N, self.M, self.K, self.V, size[self.dtype], size[self.out] if back else 0)
        # contents are whatever was there: NaN in either type
        return torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)

    def forward(self, scratch=None):
        combo.combo_grouped_cross_entropy(self.x, self.w, self.labels, self.loss, self.lse, self.begin,
                                          self.scratch(False) if scratch is None else scratch)

    def backward(self, lse, scratch=None):
        combo.combo_grouped_cross_entropy_backward(self.x, self.w, self.labels, lse, self.row_grad, self.dx, self.dw, self.begin,
                                                   self.scratch(True) if scratch is None else scratch)

    def logits(self, w):
        """Of worker w's labelled rows, and the bound of their error: K products summed, each addition off by at most a unit
        in the last place of the sum of the magnitudes."""
        a, b = self.spans[w]
        rows = torch.arange(a, b, device=DEV)[self.has[a:b]]
        x, wt = self.x[rows].double(), self.w[w].double()
        return rows, x, wt, x @ wt.T, 2 * (self.K + 4) * U * (x.abs() @ wt.abs().T)

    def check_forward(self):
        want_loss, want_lse, tol_loss, tol_lse = (torch.zeros(self.M, dtype=torch.float64, device=DEV) for _ in range(4))
        for w in range(self.N):
            rows, _, _, z, dz = self.logits(w)
            if not len(rows):
                continue
            lse = torch.logsumexp(z, 1)
            own = z.gather(1, self.labels[rows, None])[:, 0]
            # the logits' errors; an exponential's argument (at most 40 below the largest where it counts) and its own
            # error; V terms added up, at least eight side by side; the logarithm and the last sum
            d = dz.max(1).values + (200 + self.V / 8) * U + 4 * U * (lse.abs() + z.max(1).values.abs())
            want_lse[rows], want_loss[rows], tol_lse[rows], tol_loss[rows] = lse, lse - own, d, d + dz.max(1).values + 2 * U * own.abs()
        for got, want, tol, name in ((self.lse, want_lse, tol_lse, "lse"), (self.loss, want_loss, tol_loss, "loss")):
            assert (got[~self.inside] == 7.0).all(), name + " of rows of no worker was written"
            err = (got.double() - want).abs()[self.inside]
            assert not got.isnan().any() and (err <= tol[self.inside]).all(), (name, float((err / (tol[self.inside] + 1e-300)).max()))

    def exact_lse(self):
        lse = torch.zeros(self.M, device=DEV)
        for w in range(self.N):
            rows, _, _, z, _ = self.logits(w)
            if len(rows):
                lse[rows] = torch.logsumexp(z, 1).float()
        return lse

    def check_backward(self, lse):
        # d in front of the products: float weights' gradients of bfloat16 inputs keep 16 bits of it, others their type's
        half_dx = HALF[self.dtype]
        half_dw = 2.0 ** -16 if self.out != self.dtype else HALF[self.dtype]
        want_dx, tol_dx = (torch.zeros(self.M, self.K, dtype=torch.float64, device=DEV) for _ in range(2))
        for w in range(self.N):
            rows, x, wt, z, dz = self.logits(w)
            n = len(rows)
            if n:
                g = torch.full((n,), 1.0 / n, dtype=torch.float64, device=DEV) if self.row_grad is None else self.row_grad[rows].double()
                p = torch.exp(z - lse[rows].double()[:, None])
                hot = torch.zeros_like(p).scatter_(1, self.labels[rows, None], 1.0)
                d = (p - hot) * g[:, None]
                # an exponential below binary32's normal range is 0: off by less than 2^-126, whatever it is
                dd = g.abs()[:, None] * (p * (dz + (60 + 4 * (z.abs() + lse[rows].double().abs()[:, None])) * U) + 2 * U * (p + hot) + 2.0 ** -126)
                want_dx[rows] = d @ wt
                tol_dx[rows] = (dd + half_dx * d.abs()) @ wt.abs() + 2 * (self.V + 4) * U * (d.abs() @ wt.abs())
                want, tol = d.T @ x, (dd + half_dw * d.abs()).T @ x.abs() + 2 * (n + 4) * U * (d.abs().T @ x.abs())
            else:
                want, tol = (torch.zeros(self.V, self.K, dtype=torch.float64, device=DEV) for _ in range(2))
            self.near(self.dw[w], want, tol, HALF[self.out], "dw of worker %d" % w)
        self.near(self.dx[self.inside], want_dx[self.inside], tol_dx[self.inside], HALF[self.dtype], "dx")
        assert (self.dx[(~self.has) & self.inside] == 0).all()

    @staticmethod
    def near(got, want, tol, half, name):
        tol = tol + half * (want.abs() + tol) + 2.0 ** -133        # the last rounding; the smallest bfloat16
        err = (got.double() - want).abs()
        assert not got.isnan().any(), name + " is NaN"
        assert (err <= tol).all(), (name, float((err / tol).max()), float(err.max()))
