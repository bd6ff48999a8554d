"""Norms and rotation of queries and keys against their 64-bit form, element by element within the bounds that the roundings allow."""
import math

import pytest
import torch

import more_operators_reference as M
import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def make(tokens, H, K, D, dtype, dev, *, seed=0, far=1000, spread=1.0):
    gen = torch.Generator(dev).manual_seed(seed)
    qkv = (spread * torch.randn(tokens, (H + 2 * K) * D, generator=gen, device=dev)).to(dtype)
    q, k = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + K) * D].unflatten(1, (K, D))
    d_q, d_k = (torch.randn(tokens, n, D, generator=gen, device=dev).to(dtype) for n in (H, K))
    gains = [1 + 0.2 * torch.randn(D, generator=gen, device=dev) for _ in range(2)]
    positions = torch.randint(0, far, (tokens,), generator=gen, device=dev).to(torch.int32)
    return q, k, d_q, d_k, gains, positions


def within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0 and not got.isnan().any(), f"{what}: {worst} beyond the bound, at {int(off.argmax())}"


def check(op, q, k, d_q, d_k, gains, positions, fill=0.0):
    D = op.head_dim
    cos, sin = M.rotation(positions, op.rotary_dim, op.base)
    outs = [torch.full(x.shape, fill, dtype=x.dtype, device=x.device) for x in (q, k)]
    op.pm_head_norm_rotate(q, k, positions, *gains, *outs)
    dx = [torch.full(x.shape, fill, dtype=x.dtype, device=x.device) for x in (q, k)]
    dg = [torch.full((D,), fill, device=q.device) for _ in range(2)]
    op.pm_head_norm_rotate_backward(q, k, positions, *gains, d_q, d_k, *dx, *dg)
    for i, (x, d_y, name) in enumerate(((q, d_q, "q"), (k, d_k, "k"))):
        within(outs[i], *M.norm_forward(x, gains[i], cos, sin, op.interleaved, op.eps, x.dtype), name + "_out")
        want, bound, want_g, bound_g = M.norm_backward(x, gains[i], cos, sin, op.interleaved, op.eps, d_y, x.dtype)
        within(dx[i], want, bound, "d" + name)
        within(dg[i], want_g, bound_g, f"d_{name}_gain")
    return outs, dx, dg


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D,rotary", [(64, 64), (128, 128), (128, 64), (128, 0), (80, 80), (80, 48), (32, 32), (16, 16), (8, 8), (8, 4), (2, 2), (1, 0), (33, 32), (100, 100), (100, 2),
                                      (72, 40), (127, 126), (96, 32)])
def test_widths(cuda_device, D, rotary, dtype, inter):
    import paper_1910_05124_b200 as pm
    op = pm.HeadNormRotate(D, rotary_dim=rotary, interleaved=inter)
    check(op, *make(37, 3, 2, D, dtype, cuda_device, seed=D))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("tokens,H,K", [(1, 1, 1), (1, 16, 2), (2, 5, 3), (16, 16, 4), (300, 8, 8), (777, 2, 1), (5000, 2, 1), (1200, 40, 1), (3, 65, 64)])
def test_sizes(cuda_device, tokens, H, K, dtype):
    import paper_1910_05124_b200 as pm
    for D in (64, 36):
        check(pm.HeadNormRotate(D), *make(tokens, H, K, D, dtype, cuda_device, seed=tokens))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rotary", [(40, 40), (80, 40), (24, 8), (56, 56), (120, 0), (104, 24), (64, 8)])
def test_short_vectors(cuda_device, D, rotary, inter):
    """bf16 rows that vectors of 8 bytes divide and those of 16 do not, or whose strides and starts they do not."""
    import paper_1910_05124_b200 as pm
    op = pm.HeadNormRotate(D, rotary_dim=rotary, interleaved=inter)
    for tokens in (1, 301):
        check(op, *make(tokens, 5, 1, D, BF, cuda_device, seed=D + tokens))
    q, k, d_q, d_k, gains, positions = make(70, 3, 2, 64, BF, cuda_device, seed=D)
    check(pm.HeadNormRotate(64, interleaved=inter), torch.cat([q.new_zeros(70, 3, 4), q], 2)[..., 4:], k, d_q, d_k, gains, positions)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("base", [1.0, 100.0, 10000.0, 5e6])
def test_positions(cuda_device, base, dtype):
    """The smallest, the largest, and negative ones: the angle is exact everywhere."""
    import paper_1910_05124_b200 as pm
    q, k, d_q, d_k, gains, _ = make(8, 2, 1, 64, dtype, cuda_device, seed=3)
    positions = torch.tensor([0, 1, -1, 12345678, 2 ** 31 - 1, -2 ** 31, 131071, 1 << 20], dtype=torch.int32, device=cuda_device)
    for inter in (False, True):
        check(pm.HeadNormRotate(64, base=base, interleaved=inter), q, k, d_q, d_k, gains, positions)
        check(pm.HeadNormRotate(64, rotary_dim=62, base=base, interleaved=inter), q, k, d_q, d_k, gains, positions)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("spread,eps", [(1e-4, 1e-6), (1e6, 0.0), (0.0, 1e-6), (1.0, 10.0)])
def test_scales(cuda_device, spread, eps, dtype):
    import paper_1910_05124_b200 as pm
    for D in (64, 20):
        check(pm.HeadNormRotate(D, eps=eps), *make(20, 2, 2, D, dtype, cuda_device, spread=spread, seed=4))


@pytest.mark.parametrize("dtype", [BF, F])
def test_one_side_alone(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    for D in (64, 36):
        q, k, d_q, d_k, gains, positions = make(50, 4, 2, D, dtype, cuda_device, seed=5)
        op = pm.HeadNormRotate(D, rotary_dim=0)              # queries of cross attention: a norm, no rotation
        (q_out, k_out), (dq, dk), (dgq, dgk) = check(op, q, k, d_q, d_k, gains, positions)
        a, b, g = torch.zeros_like(q_out), torch.zeros_like(dq), torch.zeros_like(dgq)
        op.pm_head_norm_rotate(q, None, None, gains[0], None, a, None)
        op.pm_head_norm_rotate_backward(q, None, None, gains[0], None, d_q, None, b, None, d_q_gain=g)
        assert torch.equal(a, q_out) and torch.equal(b, dq)
        assert float((g - dgq).abs().max()) <= 1e-5 * float(dgq.abs().max())       # the groups of a token are others: another order of the sum
        a, b = torch.zeros_like(k_out), torch.zeros_like(dk)
        op.pm_head_norm_rotate(None, k, None, None, gains[1], None, a)
        op.pm_head_norm_rotate_backward(None, k, None, None, gains[1], None, d_k, None, b)     # frozen gains
        assert torch.equal(a, k_out) and torch.equal(b, dk)


@pytest.mark.parametrize("dtype", [BF, F])
def test_in_place_and_strides(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    for D in (64, 36):
        q, k, d_q, d_k, gains, positions = make(50, 4, 2, D, dtype, cuda_device, seed=6)
        op = pm.HeadNormRotate(D)
        (q_out, k_out), (dq, dk), dg = check(op, q, k, d_q, d_k, gains, positions)
        flip = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, d_q, d_k)]           # heads before tokens
        outs, dx, dg2 = check(op, *flip, gains, positions)
        assert torch.equal(outs[0], q_out) and torch.equal(dx[1], dk) and torch.equal(dg[0], dg2[0])
        odd = []
        for x in (q, k, d_q, d_k):                           # rows that no 16-byte load takes
            n, h, d = x.shape
            odd.append(torch.zeros(n * (h * d + 1) + 1, dtype=dtype, device=cuda_device).as_strided((n, h, d), (h * d + 1, d, 1), 1).copy_(x))
        check(op, *odd, gains, positions)
        gq, gk = d_q.clone(), d_k.clone()
        op.pm_head_norm_rotate_backward(q, k, positions, *gains, gq, gk, gq, gk)
        assert torch.equal(gq, dq) and torch.equal(gk, dk)
        op.pm_head_norm_rotate(q, k, positions, *gains, q, k)
        assert torch.equal(q, q_out) and torch.equal(k, k_out)


@pytest.mark.parametrize("dtype", [BF, F])
def test_values_that_are_not_finite_stay_in_their_row(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    for D in (64, 36):
        q, k, d_q, d_k, gains, positions = make(9, 4, 2, D, dtype, cuda_device, seed=7)
        op = pm.HeadNormRotate(D)
        clean, clean_dx, clean_dg = check(op, q, k, d_q, d_k, gains, positions)
        for bad in (math.nan, math.inf):
            q2 = q.clone()
            q2[4, 2, 3] = bad
            outs, dx, dg = [torch.zeros_like(x) for x in clean], [torch.zeros_like(x) for x in clean], [torch.zeros_like(x) for x in clean_dg]
            op.pm_head_norm_rotate(q2, k, positions, *gains, *outs)
            op.pm_head_norm_rotate_backward(q2, k, positions, *gains, d_q, d_k, *dx, *dg)
            keep = torch.ones(9, 4, dtype=torch.bool, device=cuda_device)
            keep[4, 2] = False
            assert torch.equal(outs[0][keep], clean[0][keep]) and torch.equal(dx[0][keep], clean_dx[0][keep]) and outs[0][4, 2].isnan().any()
            assert torch.equal(outs[1], clean[1]) and torch.equal(dx[1], clean_dx[1]) and torch.equal(dg[1], clean_dg[1])


def test_no_tokens(cuda_device):
    import paper_1910_05124_b200 as pm
    q, k, d_q, d_k, gains, positions = make(0, 2, 1, 64, BF, cuda_device)
    op = pm.HeadNormRotate(64)
    g = [torch.full((64,), 3.0, device=cuda_device) for _ in range(2)]
    op.pm_head_norm_rotate(q, k, positions, *gains, torch.zeros_like(d_q), torch.zeros_like(d_k))
    op.pm_head_norm_rotate_backward(q, k, positions, *gains, d_q, d_k, torch.zeros_like(d_q), torch.zeros_like(d_k), *g)
    assert (g[0] == 0).all() and (g[1] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_captured_replayed_and_repeated(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    q, k, d_q, d_k, gains, positions = make(200, 4, 2, 64, dtype, cuda_device, seed=8)
    q, k = q.clone(), k.clone()
    op = pm.HeadNormRotate(64)
    outs, dx, dg = [torch.zeros_like(x) for x in (q, k)], [torch.zeros_like(x) for x in (q, k)], [torch.zeros(64, device=cuda_device) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_head_norm_rotate(q, k, positions, *gains, *outs)
        op.pm_head_norm_rotate_backward(q, k, positions, *gains, d_q, d_k, *dx, *dg)
    for i in range(3):
        new = make(200, 4, 2, 64, dtype, cuda_device, seed=9 + i, far=100000)
        for x, y in zip((q, k, d_q, d_k, *gains, positions), (*new[:4], *new[4], new[5])):
            x.copy_(y)
        for x in (*outs, *dx, *dg):
            x.fill_(math.nan)
        graph.replay()
        first = [x.clone() for x in (*outs, *dx, *dg)]
        eager = check(op, q, k, d_q, d_k, gains, positions)
        assert all(torch.equal(a, b) for a, b in zip(first, [x for part in eager for x in part]))


def test_differences(cuda_device):
    """Gradients against central differences of the 64-bit form."""
    import paper_1910_05124_b200 as pm
    for inter in (False, True):
        q, k, d_q, d_k, gains, positions = make(6, 2, 1, 16, F, cuda_device, seed=12)
        op = pm.HeadNormRotate(16, rotary_dim=8, interleaved=inter)
        _, (dq, _), (dg, _) = check(op, q, k, d_q, d_k, gains, positions)
        cos, sin = M.rotation(positions, 8, op.base)
        gen = torch.Generator(cuda_device).manual_seed(13)

        def loss(x, g):
            return float((M.norm_forward(x, g, cos, sin, inter, op.eps, F)[0] * d_q.double()).sum())
        way, way_g, h = (torch.randn(s, generator=gen, device=cuda_device, dtype=torch.float64) for s in (q.shape, (16,), ())), None, 1e-6
        way, way_g, _ = way
        slope = (loss(q.double() + h * way, gains[0]) - loss(q.double() - h * way, gains[0])) / (2 * h)
        slope_g = (loss(q, gains[0].double() + h * way_g) - loss(q, gains[0].double() - h * way_g)) / (2 * h)
        assert abs(float((dq.double() * way).sum()) - slope) <= 1e-5 * float((dq.double() * way).abs().sum())
        assert abs(float((dg.double() * way_g).sum()) - slope_g) <= 1e-5 * float((dg.double() * way_g).abs().sum())
