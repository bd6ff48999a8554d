"""Norms of rows at the ends of fp32's range: beyond it on the upper side results and gradients are zeros."""
import pytest
import torch

from test_gpu_head_norm import BF, F, check, make

pytestmark = pytest.mark.gpu


# D: rows of 16-byte vectors, of 8-byte ones (bf16), and of neither
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [64, 40, 36])
@pytest.mark.parametrize("size", [1e20, 3e37, 3e38])
def test_rows_beyond_the_range(cuda_device, D, dtype, inter, size):
    """With gains above 1 even a product of two would be infinite; the other rows and sides are what they were."""
    import paper_1910_05124_b200 as pm
    q, k, d_q, d_k, gains, positions = make(9, 3, 2, D, dtype, cuda_device, seed=D)
    q, k, gains[0] = q.clone(), k.clone(), gains[0] + 2
    op = pm.HeadNormRotate(D, interleaved=inter)
    clean = check(op, q, k, d_q, d_k, gains, positions)
    other = torch.ones(9, 3, dtype=torch.bool, device=cuda_device)
    other[4, 1] = other[7, 2] = False
    q[~other] = torch.where(q[~other] < 0, -size, size).to(dtype)
    outs, dx, dg = [torch.full_like(x, 7) for x in (d_q, d_k)], [torch.full_like(x, 7) for x in (d_q, d_k)], [torch.zeros(D, device=cuda_device) for _ in range(2)]
    op.pm_head_norm_rotate(q, k, positions, *gains, *outs)
    op.pm_head_norm_rotate_backward(q, k, positions, *gains, d_q, d_k, *dx, *dg)
    for got, was in ((outs, clean[0]), (dx, clean[1])):
        assert (got[0][~other] == 0).all() and torch.equal(got[0][other], was[0][other]) and torch.equal(got[1], was[1])
    assert dg[0].isfinite().all() and torch.equal(dg[1], clean[2][1])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("spread", [1e-17, 1e17])
def test_rows_within_the_range(cuda_device, dtype, spread):
    import paper_1910_05124_b200 as pm
    for D in (64, 40, 36):
        check(pm.HeadNormRotate(D, eps=0.0), *make(20, 2, 2, D, dtype, cuda_device, spread=spread, seed=4))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("spread,small", [(1e17, 1e-6), (1e15, 1e-9), (1e-17, 1e6), (1e17, 1e6), (1e-17, 1e-12)])
def test_rows_and_gradients_of_other_sizes(cuda_device, dtype, spread, small):
    """Every product of the formula that has to be formed lies within the range."""
    import paper_1910_05124_b200 as pm
    for D in (64, 40, 36):
        q, k, d_q, d_k, gains, positions = make(20, 2, 2, D, dtype, cuda_device, spread=spread, seed=5)
        check(pm.HeadNormRotate(D, eps=0.0), q, k, d_q * small, d_k * small, gains, positions)
