"""Captured calls replayed on other inputs, and one object on two streams: every result is looked at."""
import math

import pytest
import torch

import operators_reference as R
from test_gpu_grad_clip import make as make_grads
from test_gpu_packed_attention import BF, F, make, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,K,D,lens", [(4, 2, 64, [150, 222]), (4, 4, 33, [150, 222]), (2, 1, 128, [900, 500])], ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_attention_with_other_lengths(cuda_device, dtype, H, K, D, lens):
    """The lengths are read on the device: lse, o and the three gradients of a replayed graph are those of the new ones."""
    total = sum(lens)
    op, q, k, v, d_o, cu = make(lens, H, K, D, dtype, cuda_device, seed=40)
    q, k, v = (x.clone() for x in (q, k, v))
    o, lse = torch.zeros_like(q), torch.zeros(H, total, device=cuda_device)
    g = [torch.zeros_like(x) for x in (q, k, v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_attention_packed_forward(q, k, v, cu, o, lse)
        op.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, *g)
    for i, other in enumerate(([1, total - 1], [total, 0], [0, total], [total // 2, total - total // 2])):
        new = make(other, H, K, D, dtype, cuda_device, seed=41 + i)[1:]
        for x, y in zip((q, k, v, d_o, cu), new):
            x.copy_(y)
        for x in (o, lse, *g):
            x.fill_(math.nan)
        graph.replay()
        wo, wl, bo, bl = R.attention_forward(q, k, v, cu, op.scale, True, dtype)
        within(o, wo, bo, f"o of {other}")
        within(lse, wl, bl, f"lse of {other}")
        want = R.attention_backward(q, k, v, o, lse, d_o, cu, op.scale, True, dtype)
        for x, (name, (w, b)) in zip(g, want.items()):
            within(x, w, b, f"{name} of {other}")


def clipped(grads, outs, norm, scale, max_norm):
    """The bounds of an eager call: eight squares in fp32, the rest in 64 bits, a rounding each."""
    want_norm, want_scale = R.clip(grads, max_norm)
    assert abs(float(norm) - want_norm) <= 4 * R.U32 * want_norm
    assert abs(float(scale) - want_scale) <= 5 * R.U32 * want_scale
    for g, o in zip(grads, outs):
        want = g.double() * float(scale)
        assert ((o.double() - want).abs() <= R.u(o.dtype) * want.abs() + 2.0 ** -149).all()


def test_clipping_replayed(cuda_device):
    import paper_1910_05124_b200 as pm
    g = make_grads([300000, 7, 123456, 8192], [F, BF], cuda_device, seed=42)
    outs = [torch.zeros(x.numel(), device=cuda_device) for x in g]
    norm, scale = torch.zeros(1, device=cuda_device), torch.zeros(1, device=cuda_device)
    op = pm.GradClip(g, outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_clip_gradients(100.0, norm, scale)
    for factor in (3.0, 1e-4, 5e4):                          # the norm of 431655 normal values is near 657: 1970, 0.2 and 9900
        for x in g:
            x.mul_(factor)
        for x in (norm, scale, *outs):
            x.fill_(math.nan)
        graph.replay()
        clipped(g, outs, norm, scale, 100.0)
        assert (float(scale) < 1) == (factor > 1)


def test_one_object_on_two_streams(cuda_device):
    """Two calls of one GradClip at the same time: each has a workspace of its own.  Without a limit the calls write nothing but their
    norms, in place; with outs they write the same values."""
    import paper_1910_05124_b200 as pm
    g = make_grads([3000000, 7, 123456], [F, BF], cuda_device, seed=43)
    want = R.clip(g, math.inf)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    norms, scales = ([torch.zeros(1, device=cuda_device) for _ in range(40)] for _ in range(2))
    op = pm.GradClip(g)
    torch.cuda.synchronize()
    for i in range(40):
        op.pm_clip_gradients(math.inf, norms[i], scales[i], stream=streams[i % 2])
    torch.cuda.synchronize()
    assert abs(float(norms[0]) - want) <= 4 * R.U32 * want
    assert all(torch.equal(n, norms[0]) for n in norms) and all(float(s) == 1.0 for s in scales)
