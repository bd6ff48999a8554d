"""Global norm and clipping over lists of tensors against the 64-bit form."""
import math

import pytest
import torch

import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def run(grads, max_norm, outs=None, **kw):
    import paper_1910_05124_b200 as pm
    dev = grads[0].device
    norm, scale = torch.full((1,), 9.0, device=dev), torch.full((1,), 9.0, device=dev)
    pm.GradClip(grads, outs).pm_clip_gradients(max_norm, norm, scale, **kw)
    return float(norm), float(scale)


def check(grads, max_norm, outs=None):
    want_norm, want_scale = R.clip(grads, max_norm)
    before = [g.clone() for g in grads]
    norm, scale = run(grads, max_norm, outs)
    # eight squares are added in fp32 (four roundings each), the rest in 64 bits; the root halves that; one rounding of the result
    assert abs(norm - want_norm) <= 4 * R.U32 * want_norm, (norm, want_norm)
    assert abs(scale - want_scale) <= 5 * R.U32 * want_scale
    for g, o in zip(before, grads if outs is None else outs):
        want = g.double().reshape(o.shape) * scale
        off = (o.double() - want).abs() - (R.u(o.dtype) * want.abs() + torch.finfo(o.dtype).smallest_normal * R.u(o.dtype) * 2)
        assert off.numel() == 0 or float(off.max()) <= 0
    if outs is not None:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))
    return norm, scale


def make(sizes, dtypes, dev, seed=0, spread=1.0):
    gen = torch.Generator(dev).manual_seed(seed)
    return [(spread * torch.randn(n, generator=gen, device=dev)).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


SIZES = [[1], [7], [8192], [8193, 0, 1, 8191], [100] * 40, [1000003, 5, 64], [33] * 300, [17] * 2500]


@pytest.mark.parametrize("dtypes", [[F], [BF], [F, BF]], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_in_place(cuda_device, sizes, dtypes):
    total = math.sqrt(sum(sizes))
    check(make(sizes, dtypes, cuda_device), 0.3 * total)
    g = make(sizes, dtypes, cuda_device)
    keep = [x.clone() for x in g]
    norm, scale = check(g, 30 * total)
    assert scale == 1.0 and all(torch.equal(a, b) for a, b in zip(g, keep))
    assert run(g, math.inf)[1] == 1.0


@pytest.mark.parametrize("src,dst", [([F], F), ([BF], F), ([F], BF), ([F, BF], F), ([F, BF], BF)])
@pytest.mark.parametrize("sizes", [[5, 8192, 1], [20000, 3, 8200, 0, 77]], ids=str)
def test_into_an_arena(cuda_device, sizes, src, dst):
    """Slices at multiples of 64 elements; what lies between them stays."""
    g = make(sizes, src, cuda_device, seed=1)
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // 64) * 64 + 64
    for shift in (0, 1, 3):                                  # the second and third: no 16-byte boundary anywhere
        arena = torch.full((at + 8,), 5.0, dtype=dst, device=cuda_device)
        outs = [arena[a + shift:a + shift + n] for a, n in zip(starts, sizes)]
        for max_norm in (0.1, 1e9):
            check(g, max_norm, outs)
        mask = torch.ones(at + 8, dtype=torch.bool, device=cuda_device)
        for a, n in zip(starts, sizes):
            mask[a + shift:a + shift + n] = False
        assert (arena[mask] == 5.0).all()


def test_unaligned_sources(cuda_device):
    for dtype in (F, BF):
        base = make([40000], [dtype], cuda_device, seed=2)[0]
        check([base[1:9000], base[9001:30002], base[30002:30003]], 1.0)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e-12, 1e15, 1e19, 1e30, 1e38])
def test_range(cuda_device, dtype, size):
    """Squares outside the range of fp32."""
    g = make([9000, 50], [dtype], cuda_device, seed=3)
    g = [(x.double().clamp(-3, 3) * size).to(dtype) for x in g]
    want, _ = R.clip(g, math.inf)
    if want > 3.4e38:
        assert run(g, math.inf) == (math.inf, 1.0)
        return
    norm, _ = run(g, math.inf)
    assert abs(norm - want) <= 4 * R.U32 * want + 2.0 ** -149
    check(g, want / 2)


def test_nothing_and_not_finite(cuda_device):
    z = torch.zeros(100, device=cuda_device)
    assert run([z], 1.0) == (0.0, 1.0)
    assert run([torch.zeros(0, device=cuda_device)], 1.0) == (0.0, 1.0)
    for bad, want in ((math.inf, math.inf), (-math.inf, math.inf), (math.nan, math.nan)):
        for at in (0, 9001, 20000):
            for dtype in (F, BF):
                g = make([20001], [dtype], cuda_device)[0]
                g[at] = bad
                keep = g.clone()
                out = torch.zeros_like(g)
                norm, scale = run([g], 1.0, [out])
                assert scale == 1.0 and (math.isnan(norm) if math.isnan(want) else norm == want)
                assert torch.equal(torch.nan_to_num(out, nan=3.0), torch.nan_to_num(keep, nan=3.0))


def test_more_than_32_bits_of_elements(cuda_device):
    g = torch.zeros(2 ** 32 + 77, dtype=BF, device=cuda_device)
    g[5], g[2 ** 31 + 1], g[-1] = 2.0, 4.0, 4.0
    assert run([g], 3.0) == (6.0, 0.5)
    assert (g[5], g[2 ** 31 + 1], g[-1]) == (1.0, 2.0, 2.0) and int(torch.count_nonzero(g)) == 3


def test_same_bits_streams_and_graphs(cuda_device):
    import paper_1910_05124_b200 as pm
    g = make([300000, 7, 123456], [F, BF], cuda_device, seed=4)
    outs = [torch.zeros(x.numel(), device=cuda_device) for x in g]
    op = pm.GradClip(g, outs)
    norm, scale = torch.zeros(1, device=cuda_device), torch.zeros((), device=cuda_device)
    op.pm_clip_gradients(0.5, norm, scale)
    first = [norm.clone(), scale.clone()] + [x.clone() for x in outs]
    for _ in range(3):
        op.pm_clip_gradients(0.5, norm, scale)
        assert all(torch.equal(a, b) for a, b in zip(first, [norm, scale] + outs))
    # two calls of one object at the same time: each has a workspace of its own
    streams, norms = [torch.cuda.Stream(), torch.cuda.Stream()], [torch.zeros(1, device=cuda_device) for _ in range(2)]
    ops = [pm.GradClip(g, [torch.zeros(x.numel(), device=cuda_device) for x in g]) for _ in range(2)]
    scales = [torch.zeros(1, device=cuda_device) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for o, st, n, s in zip(ops, streams, norms, scales):
            o.pm_clip_gradients(0.5, n, s, stream=st)
    torch.cuda.synchronize()
    for o, n in zip(ops, norms):
        assert torch.equal(n, first[0]) and all(torch.equal(a, b) for a, b in zip(o.outs, first[2:]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_clip_gradients(0.5, norm, scale)
    for x in g:
        x.mul_(3.0)
    graph.replay()
    want, _ = R.clip(g, 0.5)
    assert abs(float(norm) - want) <= 4 * R.U32 * want


def test_python_refusals(cuda_device):
    import paper_1910_05124_b200 as pm
    x = torch.zeros(100, device=cuda_device)
    y = torch.zeros(100, dtype=BF, device=cuda_device)
    bad = [([x], [y[:99]]), ([x], []), ([x.half()], None), ([x[::2]], None), ([x, x], None), ([x, y], [x[:100], x]), ([x[:60], x[50:]], None),
           ([y[:50]], [y[25:75]]), ([y], [x, x]), ([x[:50]], [x[25:75]]), ([x, x.cpu()], None), ([x[:10], x[10:20]], [x[10:20], x[:10]])]
    for grads, outs in bad:
        with pytest.raises(pm.PipeMareError):
            pm.GradClip(grads, outs)
    pm.GradClip([x[:50], x[50:]])
    pm.GradClip([x, x], [torch.zeros_like(x), torch.zeros_like(x)])       # read twice, written apart
    op, one = pm.GradClip([x]), torch.zeros(1, device=cuda_device)
    for a in ((0.0, one, one.clone()), (-1.0, one, one.clone()), (math.nan, one, one.clone()), (1.0, x, one), (1.0, one.double(), one)):
        with pytest.raises(pm.PipeMareError):
            op.pm_clip_gradients(*a)
