"""Tensors that are not on the GPU, and tables of the wrong type or length, are refused by the local step's calls before any
address reaches a kernel.  No GPU is needed."""
import pytest
import torch

import paper_1908_07782_b200 as combo
from paper_1908_07782_b200 import binding

HOST = "must be on the current GPU"


class Gpu:
    """Stands for a tensor on GPU 0 where nothing is asked but its place."""

    device = "cuda:0"

    def get_device(self):
        return 0


def test_products():
    x, w, y, begin = torch.zeros(4, 8), torch.zeros(2, 6, 8), torch.zeros(4, 6), torch.tensor([0, 1, 4])
    for fn, args in ((combo.combo_grouped_linear, (x, w, y, begin)), (combo.combo_grouped_linear_grad_input, (y, w, x, begin)),
                     (combo.combo_grouped_linear_grad_weight, (y, x, w, begin))):
        with pytest.raises(ValueError, match=HOST):
            fn(*args)


def test_group_norm():
    x, p = torch.zeros(3, 5, 8), torch.zeros(2, 8)
    begin, stats = torch.tensor([0, 1, 3]), torch.zeros(3, 2)
    scratch = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_group_norm(x, x.clone(), p, p, begin, 2, 1e-5, 0, stats, stats, scratch)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_group_norm_backward(x, x, x.clone(), p, p, begin, 2, 0, stats, stats, None, None, scratch)


def lists(**kw):
    a = dict(tensors=torch.zeros(3, dtype=torch.int64), begin=torch.zeros(4, dtype=torch.int64), first=torch.zeros(3, dtype=torch.int32),
             n_tensors=3, N=2, total=153, elem_bytes=4)
    a.update(kw)
    return a


def test_clipping():
    rest = dict(max_norm=1.0, norm_out=torch.zeros(2), coef_out=None, scratch=torch.zeros(1 << 14, dtype=torch.uint8))
    out = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_grad_norm(**lists(), **rest)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_grad_clip(**lists(), out=out, **rest)
    with pytest.raises(ValueError, match=HOST):
        combo.combo_check_tensors(**lists())
    for kw in (dict(tensors=torch.zeros(2, dtype=torch.int64)), dict(tensors=torch.zeros(3)), dict(begin=torch.zeros(4, dtype=torch.int32)),
               dict(begin=torch.zeros(3, dtype=torch.int64)), dict(first=torch.zeros(3, dtype=torch.int64)),
               dict(first=torch.zeros(2, dtype=torch.int32)), dict(first=torch.zeros(6, dtype=torch.int32)[::2])):
        name = "tensors and out" if "tensors" in kw else next(iter(kw))
        for fn, more in ((combo.combo_grad_norm, rest), (combo.combo_grad_clip, dict(rest, out=out)), (combo.combo_check_tensors, {})):
            with pytest.raises(ValueError, match="%s must be" % name):
                fn(**lists(**kw), **more)
    for kw in (dict(norm_out=torch.zeros(1)), dict(norm_out=torch.zeros(2).double()), dict(coef_out=torch.zeros(1))):
        with pytest.raises(ValueError, match="norm_out and coef_out must be"):
            combo.combo_grad_norm(**lists(), **dict(rest, **kw))
    with pytest.raises(ValueError, match="tensors and out must be"):
        combo.combo_grad_clip(**lists(), out=out[:2], **rest)


def test_one_on_the_host_among_others(monkeypatch):
    monkeypatch.setattr(binding, "_device", lambda: 0)
    binding._on_gpu("call", Gpu(), None, Gpu())
    for at in range(3):
        mixed = [Gpu(), Gpu()]
        mixed.insert(at, torch.zeros(1))
        with pytest.raises(ValueError, match=HOST):
            binding._on_gpu("call", *mixed)
    monkeypatch.setattr(binding, "_device", lambda: 1)
    with pytest.raises(ValueError, match=HOST):
        binding._on_gpu("call", Gpu())
