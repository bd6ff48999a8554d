"""Rows of packed attention whose every visible key has a score of -infinity: the same on every launch shape."""
import math

import pytest
import torch

from test_gpu_packed_attention import backward, forward, make

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32

# blocks of their own, and blocks that share the work of one: few heads and long sequences
SHAPES = [([450, 90], 2, 64), ([700, 40], 1, 128), ([700, 40], 40, 64), ([1500, 40], 16, 128), ([700, 40], 2, 33), ([2000, 40], 2, 64), ([60, 20], 2, 64)]


def emptied(lens, H, D, dtype, dev, n, causal):
    """The first n keys of the first sequence have scores of -infinity with every query."""
    op, q, k, v, d_o, cu = make(lens, H, H, D, dtype, dev, causal=causal, seed=21)
    clean = k.clone()
    q, k = q.clone(), k.clone()
    q[:, :, 1] = 1.0
    clean[:, :, 1] = k[:, :, 1]
    k[:n, :, 1] = -math.inf
    return op, q, clean, k, v, d_o, cu


@pytest.mark.parametrize("lens,H,D", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_causal_rows(cuda_device, dtype, lens, H, D):
    for n in (1, 5, 33, 130, 300):
        if n >= lens[0]:
            continue
        op, q, clean, k, v, d_o, cu = emptied(lens, H, D, dtype, cuda_device, n, True)
        o, lse = forward(op, q, k, v, cu)
        assert (lse[:, :n] == -math.inf).all(), (n, lse[:, :n])
        assert o[:n].isnan().all() and o[n:].isfinite().all() and lse[:, n:].isfinite().all(), n
        g = backward(op, q, k, v, o, lse, d_o, cu)
        assert g["dq"][:n].isnan().all() and g["dk"][:n].isnan().all() and g["dv"][:n].isnan().all(), n
        # the next sequence does not see it
        o0, lse0 = forward(op, q, clean, v, cu)
        g0 = backward(op, q, clean, v, o0, lse0, d_o, cu)
        a = lens[0]
        assert torch.equal(o[a:], o0[a:]) and torch.equal(lse[:, a:], lse0[:, a:])
        assert all(torch.equal(g[x][a:], g0[x][a:]) for x in g)


@pytest.mark.parametrize("lens,H,D", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_whole_sequence(cuda_device, dtype, lens, H, D):
    """Without the causal mask: every row of the sequence."""
    op, q, clean, k, v, d_o, cu = emptied(lens, H, D, dtype, cuda_device, lens[0], False)
    o, lse = forward(op, q, k, v, cu)
    a = lens[0]
    assert (lse[:, :a] == -math.inf).all() and o[:a].isnan().all()
    g = backward(op, q, k, v, o, lse, d_o, cu)
    assert all(g[x][:a].isnan().all() for x in g)
    o0, lse0 = forward(op, q, clean, v, cu)
    assert torch.equal(o[a:], o0[a:]) and torch.equal(lse[:, a:], lse0[:, a:]) and o[a:].isfinite().all()
