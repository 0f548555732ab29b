"""Refusals of the local step's calls that are answered before any device work: they need no GPU."""
import ctypes

import pytest
import torch

import paper_1908_07782_b200 as combo

INVALID, ALIAS = 1, 2


@pytest.fixture()
def place():
    """A 4 KB host buffer, 256-byte aligned: addresses that no refused call reads."""
    buf = ctypes.create_string_buffer(4096 + 256)
    a = ctypes.addressof(buf)
    yield a + (-a) % 256
    del buf


def test_scratch_sizes():
    assert combo.combo_grad_scratch_bytes(0) == 0 and combo.combo_grad_scratch_bytes(8193) == 0
    assert combo.combo_grad_scratch_bytes(8192) > combo.combo_grad_scratch_bytes(1) > 0
    assert combo.combo_group_norm_scratch_bytes(4, 0, 8, 1) == 0
    assert combo.combo_group_norm_scratch_bytes(4, 3, 8, 9) == 0
    # at least a pair of floats for each sample and channel, without a sample too
    assert combo.combo_group_norm_scratch_bytes(4, 3, 8, 2) >= 4 * 8 * 8
    assert combo.combo_group_norm_scratch_bytes(0, 3, 8, 2) > 0


def test_clipping(place):
    lib = combo.load()
    n = combo.combo_grad_scratch_bytes(2)

    def clip(t=place, o=place, b=place, f=place, T=3, N=2, total=10, e=4, m=1.0, s=place, n=n):
        return lib.combo_grad_clip(t, o, b, f, T, N, total, e, m, None, None, s, n, None)

    for kw in (dict(t=None), dict(o=None), dict(b=None), dict(f=None), dict(T=-1), dict(T=0), dict(N=0), dict(N=8193),
               dict(total=-1), dict(total=1 << 47), dict(e=8), dict(m=-0.5), dict(m=float("nan")), dict(s=None),
               dict(s=place + 4), dict(n=n - 1), dict(t=place + 4), dict(b=place + 4), dict(f=place + 2)):
        assert clip(**kw) == INVALID, kw
    # norms alone want somewhere to go
    assert lib.combo_grad_norm(place, place, place, 3, 2, 10, 4, 1.0, None, None, place, n, None) == INVALID


def test_group_norm(place):
    lib = combo.load()
    need = combo.combo_group_norm_scratch_bytes(2, 4, 8, 2)

    def norm(x=place, xp=8, y=place, yp=8, e=4, ga=place, be=place, pb=4, pp=8, begin=place, N=2, B=2, L=4, C=8, G=2, eps=1e-5,
             act=0, s=place, n=need):
        return lib.combo_group_norm(x, xp, y, yp, e, ga, be, pb, pp, begin, N, B, L, C, G, eps, act, None, None, s, n, None)

    for kw in (dict(x=None), dict(y=None), dict(xp=7), dict(yp=7), dict(e=3), dict(ga=None), dict(be=None), dict(pb=3), dict(pp=7),
               dict(begin=None), dict(begin=place + 4), dict(N=0), dict(B=-1), dict(L=0), dict(C=0), dict(G=0), dict(G=3),
               dict(eps=-1.0), dict(act=3), dict(act=-1), dict(s=None), dict(s=place + 8), dict(n=need - 1), dict(x=place + 2),
               dict(ga=place + 2)):
        assert norm(**kw) == INVALID, kw
    assert norm(B=0, x=None, y=None) == 0                     # nothing to do
    assert norm(y=place + 32) == ALIAS and norm(yp=16) == ALIAS
    wide = combo.combo_group_norm_scratch_bytes(1, 1, 4097, 1)
    assert norm(xp=4097, yp=4097, pp=4097, C=4097, G=1, B=1, L=1, n=wide) == INVALID
    back = lambda **kw: lib.combo_group_norm_backward(*[kw.get(k, v) for k, v in dict(  # noqa: E731
        dy=place, dyp=8, x=place + 512, xp=8, dx=place + 1024, dxp=8, e=4, ga=place, be=place, pb=4, pp=8, begin=place, N=2,
        B=2, L=4, C=8, G=2, act=0, mean=place, rstd=place, dg=place, db=place, gp=8, s=place, n=need, st=None).items()])
    for kw in (dict(dg=None), dict(db=None), dict(gp=7), dict(mean=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(s=None),
               dict(n=need - 1)):
        assert back(**kw) == INVALID, kw
    assert back(dx=place + 512 + 32) == ALIAS and back(dx=place + 32) == ALIAS


def test_grouped_products(place):
    lib = combo.load()
    for fn in (lib.combo_grouped_linear_grad_input, lib.combo_grouped_linear):
        def call(r1=place, p1=8, w=place + 1024, wp=8, ws=64, r2=place + 2048, p2=8, e=4, o=4, begin=place, N=2, M=4, k=8, n=8):
            return fn(r1, p1, w, wp, ws, r2, p2, e, o, begin, N, M, k, n, None)

        for kw in (dict(r1=None), dict(r2=None), dict(w=None), dict(begin=None), dict(p1=7), dict(p2=7), dict(wp=7), dict(ws=63),
                   dict(e=4, o=2), dict(e=3, o=3), dict(N=0), dict(M=-1), dict(M=(1 << 22) + 1), dict(k=0), dict(n=0), dict(r1=place + 2),
                   dict(w=place + 1026), dict(begin=place + 4)):
            assert call(**kw) == INVALID, kw
        assert call(r2=place) == ALIAS and call(r2=place + 1024) == ALIAS


def test_python_side_checks_name_what_is_wrong():
    x, w, y = torch.zeros(4, 8), torch.zeros(2, 6, 8), torch.zeros(4, 6)
    begin = torch.tensor([0, 1, 4])
    for args in ((x[:, :7], w, y, begin), (x, w, y[:3], begin), (x, w, y, begin[:2]), (x, w, y, begin.int()),
                 (x, w.transpose(1, 2).contiguous().transpose(1, 2), y, begin), (x.double(), w.double(), y, begin),
                 (x, w.bfloat16(), y, begin), (x.t().contiguous().t(), w, y, begin)):
        with pytest.raises(ValueError, match="combo_grouped_linear"):
            combo.combo_grouped_linear(*args)
    x3 = torch.zeros(3, 5, 8)
    for gamma, b, g in ((torch.zeros(2, 8), begin, 2), (torch.zeros(2, 7), begin, 2), (torch.zeros(3, 8).double(), begin, 2)):
        beta = torch.zeros(2, 8) if gamma.shape != (2, 8) else torch.zeros(3, 8)
        with pytest.raises(ValueError, match="combo_group_norm"):
            combo.combo_group_norm(x3, x3.clone(), gamma, beta, b, g, 1e-5, 0, None, None, None)
    with pytest.raises(ValueError, match="channels must be neighbours"):
        combo.combo_group_norm(x3.transpose(1, 2), x3.transpose(1, 2).clone(), None, None, None, 1, 1e-5, 0, None, None, None)
