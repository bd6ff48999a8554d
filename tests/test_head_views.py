"""Tensors that a call with heads writes: the check of their strides is the one that every such call makes."""
from types import SimpleNamespace

import pytest
import torch

import paper_1910_05124_b200 as pm

HOST = SimpleNamespace(index=-1)                  # what get_device() gives for these tensors


@pytest.mark.parametrize("make", [lambda: pm.PackedAttention(4, 2, 8), lambda: pm.CrossAttention(4, 2, 8), lambda: pm.HeadNormRotate(8)])
def test_written_tensors_are_checked(make, monkeypatch):
    from paper_1910_05124_b200 import build
    build.build()
    op, seen = make(), []
    check = type(op)._check_apart
    monkeypatch.setattr(type(op), "_check_apart", lambda self, name, dims: (seen.append(name), check(self, name, dims)))
    shape, plain, shared = (5, 4, 8), torch.zeros(5, 4, 8), torch.zeros(1, 4, 8).expand(5, 4, 8)
    apart = torch.zeros(4, 5, 8).transpose(0, 1)
    views = op._views((shape, None, shape, shape), torch.float32, HOST, ("q", "k", "o", "p"), (shared, None, plain, apart), 1)
    assert views[1] is None and len(views) == 4 and seen == ["p"]
    with pytest.raises(pm.PipeMareError, match="o overlaps itself"):
        op._views((shape, shape), torch.float32, HOST, ("q", "o"), (plain, shared), 1)
