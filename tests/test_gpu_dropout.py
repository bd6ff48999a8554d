"""Dropout against the generator's definition: which elements are kept, and their values within the roundings."""
import math

import pytest
import torch

import more_operators_reference as M
import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def rng_of(dev, seed=99, first=12345):
    return torch.tensor([seed, first], dtype=torch.int64, device=dev)


def within(got, x, residual, mask, scale):
    """The product's rounding, the sum's, and the result's."""
    kept = torch.where(mask, x.double() * scale, 0.0)
    want = kept if residual is None else kept + residual.double()
    bound = 2 * R.U32 * kept.abs() + R.U32 * want.abs() + R.u(got.dtype) * want.abs() * (1 + 2.0 ** -7) + R.TINY
    assert ((got.double() - want).abs() <= bound).all() and not got.isnan().any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (96, 200), (33, 129), (4097,), (5000, 71), (2, 3, 4)], ids=str)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_values(cuda_device, shape, p, dtype):
    import paper_1910_05124_b200 as pm
    gen = torch.Generator(cuda_device).manual_seed(1)
    x, res, d_y = (torch.randn(shape, generator=gen, device=cuda_device).to(dtype) for _ in range(3))
    op, rng, n = pm.Dropout(p), rng_of(cuda_device), x.numel()
    mask, scale = M.kept(n, p, 99, 12345)
    mask = mask.to(cuda_device).view(shape)
    for residual in (None, res):
        y = torch.full_like(x, math.nan)
        op.pm_dropout(x, rng, y, residual=residual)
        within(y, x, residual, mask, scale)
    d_x = torch.full_like(x, math.nan)
    op.pm_dropout_backward(d_y, rng, d_x)
    within(d_x, d_y, None, mask, scale)
    if p == 0.0:
        assert torch.equal(d_x, d_y)


@pytest.mark.parametrize("seed,first", [(0, 0), (-1, -1), (-2 ** 63, 2 ** 63 - 1), (1 << 32, (1 << 32) - 3), ((1 << 63) - 1, -3)])
def test_keys_and_counters(cuda_device, seed, first):
    """Both numbers are taken as 64 bits; counters pass 32 bits and wrap at 64."""
    import paper_1910_05124_b200 as pm
    x = torch.ones(200, device=cuda_device)
    y = torch.zeros_like(x)
    pm.Dropout(0.5).pm_dropout(x, rng_of(cuda_device, seed, first), y)
    mask, _ = M.kept(200, 0.5, seed, first)
    assert torch.equal(y != 0, mask.to(cuda_device))


@pytest.mark.parametrize("dtype", [BF, F])
def test_dropped_values_may_be_anything(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    n = 5003
    mask = M.kept(n, 0.5, 99, 12345)[0].to(cuda_device)
    x = torch.ones(n, device=cuda_device).to(dtype)
    x[~mask] = torch.tensor([math.nan, math.inf], device=cuda_device).to(dtype).repeat(n)[:int((~mask).sum())]
    res = torch.full_like(x, 2.0)
    y = torch.zeros_like(x)
    pm.Dropout(0.5).pm_dropout(x, rng_of(cuda_device), y, residual=res)
    assert (y[mask] == 4).all() and (y[~mask] == 2).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_in_place_and_odd_starts(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    gen = torch.Generator(cuda_device).manual_seed(2)
    n, op, rng = 10007, pm.Dropout(0.2), rng_of(cuda_device)
    x, res = (torch.randn(n, generator=gen, device=cuda_device).to(dtype) for _ in range(2))
    y = torch.zeros_like(x)
    op.pm_dropout(x, rng, y, residual=res)
    for start in (1, 2, 3):                                  # no 16-byte boundary
        a, b, c = (torch.zeros(n + 8, dtype=dtype, device=cuda_device) for _ in range(3))
        a[start:start + n], b[start:start + n] = x, res
        op.pm_dropout(a[start:start + n], rng, c[start:start + n], residual=b[start:start + n])
        assert torch.equal(c[start:start + n], y) and (c[:start] == 0).all() and (c[start + n:] == 0).all()
    for into in (x, res):
        a, b = x.clone(), res.clone()
        op.pm_dropout(a, rng, a if into is x else b, residual=b)
        assert torch.equal(a if into is x else b, y)


def test_replays_draw_anew(cuda_device):
    """The generator's numbers are read on the device: a replay after they have moved on draws others, the backward call the same."""
    import paper_1910_05124_b200 as pm
    n, op = 4096, pm.Dropout(0.3)
    x, y, d = torch.ones(n, device=cuda_device), torch.zeros(n, device=cuda_device), torch.zeros(n, device=cuda_device)
    rng = rng_of(cuda_device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_dropout(x, rng, y)
        op.pm_dropout_backward(x, rng, d)
        rng[1].add_(op.counters(n))
    first = 12345
    for _ in range(3):
        graph.replay()
        mask = M.kept(n, 0.3, 99, first)[0].to(cuda_device)
        assert torch.equal(y != 0, mask) and torch.equal(y, d)
        first += n // 8
    assert rng.tolist() == [99, first]


def test_share_of_kept_elements(cuda_device):
    """Over 2^22 elements the share kept is within six standard deviations, and neighbours and halves of a word are independent."""
    import paper_1910_05124_b200 as pm
    n, p = 1 << 22, 0.1
    x, y = torch.ones(n, device=cuda_device), torch.zeros(n, device=cuda_device)
    pm.Dropout(p).pm_dropout(x, rng_of(cuda_device), y)
    kept = (y != 0).double()
    assert abs(float(kept.mean()) - (1 - p)) <= 6 * math.sqrt(p * (1 - p) / n) + 2.0 ** -17
    for lag in (1, 2, 8, 16):
        both = float((kept[lag:] * kept[:-lag]).mean())
        assert abs(both - (1 - p) ** 2) <= 6 * math.sqrt((1 - p) ** 2 / n) + 2.0 ** -15


def test_more_than_32_bits_of_elements(cuda_device):
    import paper_1910_05124_b200 as pm
    n = (1 << 32) + 4099
    x = torch.ones(n, dtype=BF, device=cuda_device)
    rng = rng_of(cuda_device)
    pm.Dropout(0.5).pm_dropout(x, rng, x)
    for at in (0, (1 << 31) - 64, (1 << 32) - 64, (1 << 32) + 4000):
        part = x[at:at + 99]
        mask = M.kept(part.numel(), 0.5, 99, 12345 + at // 8)[0].to(cuda_device)
        assert at % 8 == 0 and torch.equal(part != 0, mask) and (part[mask] == 2).all()
