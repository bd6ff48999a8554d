"""Gradient clipping where the norm or the factor leaves the range of fp32."""
import math

import pytest
import torch

import operators_reference as R
from test_gpu_grad_clip import make, run

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
PAIRS = [(F, F, True), (BF, BF, True), (F, F, False), (BF, F, False), (F, BF, False), (BF, BF, False)]
IDS = [f"{str(s)[6:]}-{str(d)[6:]}-{'in_place' if i else 'apart'}" for s, d, i in PAIRS]


@pytest.mark.parametrize("src,dst,in_place", PAIRS, ids=IDS)
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e30, 1e39])
def test_norm_above_the_range_of_fp32(cuda_device, src, dst, in_place, max_norm):
    """9000 gradients near 1e38: a norm near 1e40 is reported as infinity, and an infinite norm scales nothing."""
    g = [(x.double().clamp(-3, 3) * 1e38).to(src) for x in make([9000, 50, 8192], [src], cuda_device, seed=6)]
    keep = [x.clone() for x in g]
    outs = None if in_place else [torch.zeros(x.numel(), dtype=dst, device=cuda_device) for x in g]
    assert R.clip(g, math.inf)[0] > 3.5e38
    assert run(g, max_norm, outs) == (math.inf, 1.0)
    for a, b in zip(keep, g if in_place else outs):
        assert torch.equal(a.to(dst), b)


@pytest.mark.parametrize("src,dst,in_place", PAIRS, ids=IDS)
@pytest.mark.parametrize("size,max_norm", [(1e36, 1e-6), (1e36, 1e-10), (1e34, 1e-4), (1e30, 1e-12), (1e36, 1e-30), (1e20, 1e-30), (1.0, 1e-44), (1e36, 1e-50), (1.0, 1e-300)])
def test_factor_below_the_normal_range_of_fp32(cuda_device, src, dst, in_place, size, max_norm):
    """The factor itself has few bits there, or none; what it scales has them all."""
    g = [(x.double().clamp(-3, 3) * size).to(src) for x in make([9000, 50, 8192], [src], cuda_device, seed=7)]
    want_norm, want_scale = R.clip(g, max_norm)
    before = [x.clone() for x in g]
    outs = None if in_place else [torch.zeros(x.numel(), dtype=dst, device=cuda_device) for x in g]
    norm, scale = run(g, max_norm, outs)
    assert abs(norm - want_norm) <= 4 * R.U32 * want_norm
    assert abs(scale - want_scale) <= 5 * R.U32 * want_scale + 2.0 ** -150
    for a, b in zip(before, g if in_place else outs):
        want = a.double() * want_scale
        # the norm's error, the 64-bit factor's, the rounding to fp32 and that to the result's type; below 2^-126 halves of the smallest steps
        bound = (4 * R.U32 + R.U32 + 2.0 ** -50 + R.u(dst)) * want.abs() + 2.0 ** -150 + torch.finfo(dst).smallest_normal * R.u(dst)
        off = (b.double() - want).abs() - bound
        assert float(off.max()) <= 0, float(off.max())


def test_norm_and_scale_lie_apart_from_the_tensors(cuda_device):
    """Within the arena, but between its slices, they may lie."""
    import paper_1910_05124_b200 as pm
    arena, g = torch.zeros(1000, device=cuda_device), make([100, 0, 200], [F, BF], cuda_device, seed=8)
    outs = [arena[0:100], arena[128:128], arena[128:328]]
    op, one = pm.GradClip(g, outs), torch.zeros(1, device=cuda_device)
    for bad in (arena[0:1], arena[99:100], arena[327:328], g[0][50:51], g[2].view(F)[40:41] if g[2].dtype == BF else g[2][40:41]):
        with pytest.raises(pm.PipeMareError, match="norm lies in"):
            op.pm_clip_gradients(1.0, bad, one)
        with pytest.raises(pm.PipeMareError, match="scale lies in"):
            op.pm_clip_gradients(1.0, one, bad)
    assert (arena == 0).all()
    op.pm_clip_gradients(1.0, arena[100:101], arena[328:329])
    want = R.clip(g, 1.0)
    assert abs(float(arena[100]) - want[0]) <= 4 * R.U32 * want[0] and abs(float(arena[328]) - want[1]) <= 5 * R.U32 * want[1]
    empty = pm.GradClip([torch.zeros(0, device=cuda_device)])
    empty.pm_clip_gradients(1.0, one, arena[500:501])
    assert float(one) == 0.0 and float(arena[500]) == 1.0
