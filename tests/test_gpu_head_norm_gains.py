"""The gains' gradients as whole numbers: a row that is left out, or counted twice, changes every one of them by one."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rotary", [0, 64])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,H,K", [(1, 3, 1), (1200, 40, 1), (777, 16, 2), (12291, 5, 3), (3, 65, 64)])
def test_every_row_counts_once(cuda_device, tokens, H, K, dtype, aligned, rotary):
    """Rows and gradients of +-1, positions of 0: r is 1, and each row adds +-1 to each sum.  r is off by two units in the last place at most, so
    61455 rows are off by 2^-22 each, 0.015 in all; sums of whole numbers below 2^24 are exact."""
    import paper_1910_05124_b200 as pm
    D, gen = 64, torch.Generator(cuda_device).manual_seed(tokens)
    pad = 0 if aligned else 1                     # rows that start at no vector take the kernel of any layout

    def signs(heads):
        x = torch.randint(0, 2, (tokens, heads, D + pad), generator=gen, device=cuda_device) * 2 - 1
        return x.to(dtype)[..., pad:]
    q, k, d_q, d_k = signs(H), signs(K), signs(H), signs(K)
    ones, positions = torch.ones(D, device=cuda_device), torch.zeros(tokens, dtype=torch.int32, device=cuda_device)
    op = pm.HeadNormRotate(D, rotary_dim=rotary, eps=0.0)
    for gains in ((0,), (1,), (0, 1)):            # both sides, and either alone: other numbers of blocks
        got = [torch.zeros(D, device=cuda_device) for _ in range(2)]
        side = [(q, d_q, torch.zeros(tokens, H, D, dtype=dtype, device=cuda_device)), (k, d_k, torch.zeros(tokens, K, D, dtype=dtype, device=cuda_device))]
        x, dy, dx = zip(*[s if i in gains else (None,) * 3 for i, s in enumerate(side)])
        g, dg = zip(*[(ones, got[i]) if i in gains else (None, None) for i in range(2)])
        op.pm_head_norm_rotate_backward(*x, positions, *g, *dy, *dx, *dg)
        for i in gains:
            want = (side[i][0].double() * side[i][1].double()).sum((0, 1))
            assert float((got[i].double() - want).abs().max()) < 0.25
