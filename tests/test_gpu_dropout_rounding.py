"""The roundings of dropout as documented, bit for bit: the scale to fp32, product and sum in one, a bf16 result from that."""
import numpy as np
import pytest
import torch

import more_operators_reference as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p", [0.1, 0.3, 0.5, 0.999])
def test_bits(cuda_device, p, dtype):
    """Values of 8 bits, so that the product (24 + 8 bits) and the sum (within 53) are exact in 64 bits and rounding that is the fused result."""
    import paper_1910_05124_b200 as pm
    n, gen = 5003, torch.Generator().manual_seed(int(1000 * p))
    x, res = (torch.randint(-255, 256, (n,), generator=gen).double() * 2.0 ** torch.randint(-4, 5, (n,), generator=gen).double() for _ in range(2))
    mask, scale = M.kept(n, p, 99, 12345)
    scale32 = float(np.float32(scale))
    y, rng = torch.zeros(n, dtype=dtype, device=cuda_device), torch.tensor([99, 12345], device=cuda_device)
    for residual in (None, res):
        pm.Dropout(p).pm_dropout(x.to(cuda_device, dtype), rng, y, residual=None if residual is None else residual.to(cuda_device, dtype))
        want = torch.where(mask, x * scale32, 0.0) + (0.0 if residual is None else residual)
        assert torch.equal(y.cpu(), want.float().to(dtype))
