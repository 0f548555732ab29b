"""Refusals of the grouped cross entropy and of dropout that are answered before any device work: they need no GPU."""
import ctypes

import pytest
import torch

import paper_1908_07782_b200 as combo

INVALID, ALIAS = 1, 2
HOST = "must be on the current GPU"


@pytest.fixture()
def place():
    """A 64 KB host buffer, 256-byte aligned: addresses that no refused call reads."""
    buf = ctypes.create_string_buffer(65536 + 256)
    a = ctypes.addressof(buf)
    yield a + (-a) % 256
    del buf


def scratch(*a):
    return combo.combo_grouped_cross_entropy_scratch_bytes(*a)


def test_scratch_sizes():
    for bad in ((0, 4, 8, 8, 4, 0), (8193, 4, 8, 8, 4, 0), (2, -1, 8, 8, 4, 0), (2, (1 << 22) + 1, 8, 8, 4, 0), (2, 4, 0, 8, 4, 0),
                (2, 4, 8, 0, 4, 0), (2, 4, (1 << 20) + 1, 8, 4, 0), (2, 4, 8, (1 << 20) + 1, 4, 0), (2, 4, 8, 8, 3, 0), (2, 4, 8, 8, 4, 2),
                (2, 4, 8, 8, 2, 8)):
        assert scratch(*bad) == 0, bad
    for elem, grad in ((4, 0), (4, 4), (2, 0), (2, 2), (2, 4)):
        assert scratch(2, 0, 8, 8, elem, grad) > 0
        assert scratch(2, 100, 64, 1000, elem, grad) >= scratch(2, 4, 64, 1000, elem, grad) > 0


def test_cross_entropy(place):
    lib = combo.load()
    at = lambda k: place + 2048 * k  # noqa: E731
    need = scratch(2, 4, 8, 8, 4, 0)
    base = dict(x=at(0), xp=8, w=at(1), wp=8, ws=64, e=4, lab=at(2), begin=at(3), N=2, M=4, k=8, n=8, loss=at(4), lse=at(5), s=at(10), b=need, st=None)

    def call(**kw):
        return lib.combo_grouped_cross_entropy(*dict(base, **kw).values())

    for kw in (dict(x=None), dict(w=None), dict(lab=None), dict(begin=None), dict(loss=None), dict(lse=None), dict(s=None), dict(xp=7),
               dict(wp=7), dict(ws=63), dict(e=3), dict(N=0), dict(N=8193), dict(M=-1), dict(M=(1 << 22) + 1), dict(k=0), dict(n=0),
               dict(k=(1 << 20) + 1), dict(n=(1 << 20) + 1), dict(b=need - 1), dict(s=at(10) + 128), dict(x=at(0) + 2), dict(w=at(1) + 2),
               dict(lab=at(2) + 4), dict(begin=at(3) + 4), dict(loss=at(4) + 2), dict(lse=at(5) + 1), dict(xp=1 << 40), dict(ws=1 << 44)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(loss=at(5)), dict(loss=at(0)), dict(lse=at(1)), dict(loss=at(2)), dict(lse=at(3)), dict(loss=at(10)), dict(s=at(1)),
               dict(s=at(2))):
        assert call(**kw) == ALIAS, kw


def test_cross_entropy_backward(place):
    lib = combo.load()
    at = lambda k: place + 2048 * k  # noqa: E731
    need = scratch(2, 4, 8, 8, 4, 4)
    base = dict(x=at(0), xp=8, w=at(1), wp=8, ws=64, e=4, lab=at(2), lse=at(3), g=at(4), dx=at(5), dxp=8, dw=at(6), dwp=8, dws=64, o=4,
                begin=at(7), N=2, M=4, k=8, n=8, s=at(10), b=need, st=None)

    def call(**kw):
        return lib.combo_grouped_cross_entropy_backward(*dict(base, **kw).values())

    for kw in (dict(x=None), dict(w=None), dict(lab=None), dict(begin=None), dict(lse=None), dict(dx=None), dict(dw=None), dict(s=None),
               dict(xp=7), dict(wp=7), dict(ws=63), dict(dxp=7), dict(dwp=7), dict(dws=63), dict(e=3), dict(o=2), dict(o=0), dict(e=2, o=3),
               dict(N=0), dict(M=-1), dict(k=0), dict(n=0), dict(b=need - 1), dict(s=at(10) + 128), dict(dx=at(5) + 2), dict(dw=at(6) + 2),
               dict(lse=at(3) + 2), dict(g=at(4) + 2)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(dx=at(0)), dict(dx=at(0) + 32), dict(dx=at(1)), dict(dw=at(1)), dict(dw=at(0)), dict(dx=at(6)), dict(dw=at(2)),
               dict(dx=at(3)), dict(dx=at(4)), dict(dw=at(7)), dict(s=at(6)), dict(s=at(0))):
        assert call(**kw) == ALIAS, kw


def test_dropout(place):
    lib = combo.load()
    base = dict(x=place, xp=8, r=None, rp=0, y=place + 4096, yp=8, e=4, begin=place + 8192, N=2, M=4, n=8, p=0.5, seed=1, rnd=2, site=3, first=0,
                st=None)

    def call(**kw):
        return lib.combo_dropout(*dict(base, **kw).values())

    for kw in (dict(x=None), dict(y=None), dict(xp=7), dict(yp=7), dict(r=place + 2048, rp=7), dict(e=3), dict(begin=None),
               dict(begin=place + 4), dict(N=0), dict(N=8193), dict(M=-1), dict(n=0), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")),
               dict(first=-1), dict(first=8191), dict(x=place + 2), dict(y=place + 2), dict(r=place + 2050, rp=8), dict(n=1 << 33),
               dict(M=1 << 40)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(y=place + 32), dict(y=place, yp=16), dict(r=place + 4096 + 32, rp=8), dict(r=place + 4096, rp=16)):
        assert call(**kw) == ALIAS, kw


def test_python_side_checks_name_what_is_wrong():
    x, w, y = torch.zeros(4, 8), torch.zeros(2, 6, 8), torch.zeros(4, dtype=torch.int64)
    begin, f, s = torch.tensor([0, 1, 4]), torch.zeros(4), torch.zeros(4096, dtype=torch.uint8)
    for args in ((x[:, :7], w, y, f, f, begin, s), (x, w, y[:3], f, f, begin, s), (x, w, y.int(), f, f, begin, s), (x, w, y, f[:3], f, begin, s),
                 (x, w, y, f, f.double(), begin, s), (x, w, y, f, f, begin[:2], s), (x, w, y, f, f, begin.int(), s),
                 (x.double(), w.double(), y, f, f, begin, s), (x, w.bfloat16(), y, f, f, begin, s), (x.t().contiguous().t(), w, y, f, f, begin, s),
                 (x, w.transpose(1, 2).contiguous().transpose(1, 2), y, f, f, begin, s), (x, w[0], y, f, f, begin, s)):
        with pytest.raises(ValueError, match="combo_grouped_cross_entropy"):
            combo.combo_grouped_cross_entropy(*args)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_grouped_cross_entropy(x, w, y, f, f, begin, s)
    for dx, dw in ((x[:3], w), (x.bfloat16(), w), (x, w[:1]), (x, w.double()), (x, w.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError, match="combo_grouped_cross_entropy_backward: d"):
            combo.combo_grouped_cross_entropy_backward(x, w, y, f, None, dx, dw, begin, s)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_grouped_cross_entropy_backward(x, w, y, f, None, x.clone(), w.clone(), begin, s)
    for kw in (dict(x=x.double()), dict(y=x[:3]), dict(residual=x.bfloat16()), dict(begin=begin.int()), dict(seed=1 << 64), dict(rnd=-1),
               dict(site=1 << 32), dict(x=x.t().contiguous().t())):
        with pytest.raises(ValueError, match="combo_dropout"):
            combo.combo_dropout(**dict(dict(x=x, residual=None, y=x.clone(), begin=begin, p=0.5, seed=1, rnd=0), **kw))
    with pytest.raises(ValueError, match=HOST):
        combo.combo_dropout(x, None, x.clone(), begin, 0.5, 1, 0)


def test_least_scratch(place):
    """Less scratch than asked for is taken, down to the least; it is far less than all rows' logits where those are large."""
    least = combo.combo_grouped_cross_entropy_least_scratch_bytes
    assert least(2, 4, 8, 8, 4, 2) == 0 and least(2, -1, 8, 8, 4, 0) == 0
    for elem, grad in ((4, 0), (4, 4), (2, 0), (2, 2), (2, 4)):
        for N, M, k, v in ((2, 4, 8, 8), (8, 6536, 1024, 30001), (64, 64, 1000, 4500), (1024, 4096, 512, 10), (1, 1 << 22, 64, 1 << 20)):
            assert 0 < least(N, M, k, v, elem, grad) <= scratch(N, M, k, v, elem, grad)
        # the weights, the rows and an eighth of their logits
        assert least(8, 6536, 1024, 30001, elem, grad) < 6536 * 30001 * 4 // 4
    # a copy of bfloat16 weights, which a call on 16-byte boundaries does not make, takes a quarter of a gigabyte at most
    assert scratch(16, 16, 1024, 32000, 2, 0) < 300 << 20 and least(16, 16, 1024, 32000, 2, 0) < 16 << 20
    # few classes: the weights' three planes, not those of a tile's 128 classes
    assert scratch(1024, 1024, 4096, 10, 4, 4) < 6 * (1024 * 16 + 1024 * 64 + 128) * 4096 + 4 * 1024 * 64 * 4096 + (64 << 20)
    lib = combo.load()
    at = lambda k: place + 2048 * k  # noqa: E731
    need = least(2, 3000, 64, 1000, 2, 0)
    assert lib.combo_grouped_cross_entropy(at(0), 64, at(1), 64, 64000, 2, at(2), at(3), 2, 3000, 64, 1000, at(4), at(5), at(10), need - 1, None) == INVALID


def test_dropout_refuses_to_write_over_its_table(place):
    lib = combo.load()
    for begin in (place + 4096, place + 4096 + 8 * 3, place + 4096 - 16, place + 4096 + 120):
        # y: four rows of eight floats, 128 bytes from place + 4096 on; begin: 24 bytes
        assert lib.combo_dropout(place, 8, None, 0, place + 4096, 8, 4, begin, 2, 4, 8, 0.5, 1, 2, 3, 0, None) == ALIAS, begin - place
