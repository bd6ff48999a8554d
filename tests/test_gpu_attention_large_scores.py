"""Scores up to 2^30 in size, whole numbers that every kernel forms exactly: the rows are the means of the largest keys' values, and finite."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# single tokens, beams, tiles of heads up to 64 in blocks that stay and in blocks of their own, heads of 128 alike, CUDA-core layouts
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lens,kv,H,K,D", [([1, 1, 2], [700, 33, 1], 4, 4, 64), ([4, 3], [300, 1000], 8, 2, 128), ([200, 90], [300, 129], 2, 2, 64), ([130] * 40, [77] * 40, 8, 8, 64),
                                           ([200, 90], [300, 129], 2, 1, 128), ([1000] * 4, [150] * 4, 16, 8, 128), ([50, 70], [300, 129], 2, 1, 36)])
def test_forward(cuda_device, lens, kv, H, K, D, sign, dtype):
    """q = 2^13 in one dimension, k = sign 2^13 n there: s = sign 2^26 n for n up to 16.  Exponentials of what is 2^26 below the maximum are zero."""
    import paper_1910_05124_b200 as pm
    gen = torch.Generator(cuda_device).manual_seed(D + len(lens))
    T, S = sum(lens), sum(kv)
    q, k = torch.zeros(T, H, D, device=cuda_device), torch.zeros(S, K, D, device=cuda_device)
    n = torch.randint(1, 17, (S, K), generator=gen, device=cuda_device)
    q[..., 5], k[..., 5] = 2.0 ** 13, sign * 2.0 ** 13 * n
    v = torch.randint(-8, 9, (S, K, D), generator=gen, device=cuda_device).float()
    starts = [torch.tensor([sum(x[:i]) for i in range(len(x) + 1)], dtype=torch.int32, device=cuda_device) for x in (lens, kv)]
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    o, lse = torch.zeros_like(q), torch.zeros(H, T, device=cuda_device)
    pm.CrossAttention(H, K, D, scale=1.0).pm_attention_cross_forward(q, k, v, *starts, o, lse)
    u = torch.finfo(dtype).eps / 2
    for b, (x, y) in enumerate(zip(lens, kv)):
        t0, s0 = int(starts[0][b]), int(starts[1][b])
        for h in range(H):
            score = sign * n[s0:s0 + y, h // (H // K)]
            top = score == score.max()
            want = v[s0:s0 + y, h // (H // K)][top].double().mean(0)
            got = o[t0:t0 + x, h].double()
            # the quotient of two sums that are exact but for a common factor's rounding (P in bf16: u), and the result's rounding
            assert ((got - want).abs() <= 3 * u * v[s0:s0 + y, h // (H // K)][top].double().abs().mean(0) + 2 * u * want.abs()).all()
            assert ((lse[h, t0:t0 + x].double() - float(score.max()) * 2.0 ** 26).abs() <= 2.0 ** 30 * 2.0 ** -22).all()
