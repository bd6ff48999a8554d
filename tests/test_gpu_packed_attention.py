"""Attention over packed sequences against its 64-bit form, element by element within the bounds that the roundings allow."""
import math

import pytest
import torch

import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def make(lens, H, K, D, dtype, dev, *, first=0, tail=0, causal=True, seed=0, scale=None, spread=1.0):
    import paper_1910_05124_b200 as pm
    gen = torch.Generator(dev).manual_seed(seed)
    T = first + sum(lens) + tail
    qkv = (spread * torch.randn(T, (H + 2 * K) * D, generator=gen, device=dev)).to(dtype)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([H * D, K * D, K * D], 1))
    d_o = torch.randn(T, H, D, generator=gen, device=dev).to(dtype)
    cu = R.lens_to_cu(lens, dev, first)
    op = pm.PackedAttention(H, K, D, causal=causal, scale=scale)
    return op, q, k, v, d_o, cu


def forward(op, q, k, v, cu, fill=0.0, **kw):
    o = torch.full(q.shape, fill, dtype=q.dtype, device=q.device)
    lse = torch.full((q.shape[1], q.shape[0]), fill, device=q.device)
    op.pm_attention_packed_forward(q, k, v, cu, o, lse, **kw)
    return o, lse


def backward(op, q, k, v, o, lse, d_o, cu, fill=0.0, **kw):
    # one buffer for the three gradients, as the projection's backward pass wants it
    T, H, D = q.shape
    K = k.shape[1]
    buf = torch.full((T, (H + 2 * K) * D), fill, dtype=q.dtype, device=q.device)
    g = [x.unflatten(1, (-1, D)) for x in buf.split([H * D, K * D, K * D], 1)]
    op.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, *g, **kw)
    return dict(zip(("dq", "dk", "dv"), g))


def within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0 and not got.isnan().any(), f"{what}: {worst} beyond the bound, at {int(off.argmax())}"


def check(op, q, k, v, d_o, cu):
    o, lse = forward(op, q, k, v, cu)
    wo, wl, bo, bl = R.attention_forward(q, k, v, cu, op.scale, op.causal, q.dtype)
    within(o, wo, bo, "o")
    within(lse, wl, bl, "lse")
    got = backward(op, q, k, v, o, lse, d_o, cu)
    for name, (want, bound) in R.attention_backward(q, k, v, o, lse, d_o, cu, op.scale, op.causal, q.dtype).items():
        within(got[name], want, bound, name)


LENS = [[1], [2, 1, 3], [17, 1, 46], [64], [65, 63], [127, 128, 129], [200, 0, 5, 300], [256, 255, 257, 1], [700, 31], [1030], [512, 897, 640]]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths(cuda_device, lens, dtype, causal):
    check(*make(lens, 2, 1, 64, dtype, cuda_device, causal=causal))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [1, 7, 8, 24, 32, 33, 56, 64, 72, 80, 96, 120, 128])
def test_head_widths(cuda_device, D, dtype):
    check(*make([130, 70], 2, 2, D, dtype, cuda_device, seed=D))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (8, 2), (5, 5), (16, 1)])
def test_shared_heads(cuda_device, H, K, dtype):
    check(*make([40, 150], H, K, 128 if H < 8 else 64, dtype, cuda_device, seed=H))
    if H < 16:
        check(*make([1100], H, K, 64 if H < 8 else 128, dtype, cuda_device, seed=H))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [30, 32, 61, 64, 100, 128])
def test_many_heads(cuda_device, D, dtype):
    """More blocks than run at a time."""
    check(*make([130, 257, 64], 40, 8, D, dtype, cuda_device, seed=D))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,H,K,D", [([2000], 2, 1, 64), ([1500, 3], 1, 1, 64), ([1300], 2, 2, 128), ([1, 900], 4, 1, 120), ([700], 1, 1, 33),
                                        ([3000], 1, 1, 8)], ids=str)
def test_few_blocks(cuda_device, lens, H, K, D, dtype, causal):
    """Long sequences and few heads: blocks share the work of one."""
    check(*make(lens, H, K, D, dtype, cuda_device, causal=causal, first=3, tail=50, seed=len(lens) + D))


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_sequences(cuda_device, dtype):
    lens = [(7 * i) % 23 for i in range(300)]                # more sequences than one round of the tile search takes, empty ones too
    check(*make(lens, 2, 1, 32, dtype, cuda_device, seed=1))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("spread,scale", [(6.0, None), (0.01, None), (1.0, 2.0)])
def test_peaked_and_flat_scores(cuda_device, dtype, spread, scale):
    check(*make([300], 2, 1, 64, dtype, cuda_device, spread=spread, scale=scale, seed=2))


@pytest.mark.parametrize("dtype", [BF, F])
def test_growing_scores(cuda_device, dtype):
    """Every key tile raises the running maximum by far, so that all sums are rescaled every time; then the reverse."""
    op, q, k, v, d_o, cu = make([520], 2, 1, 64, dtype, cuda_device, seed=3, scale=0.5)
    ramp = torch.linspace(0.1, 8, 520, device=cuda_device)
    for r in (ramp, ramp.flip(0)):
        k2 = (k.float().abs() * r[:, None, None]).to(dtype)
        check(op, q.abs(), k2, v, d_o, cu)


@pytest.mark.parametrize("dtype", [BF, F])
def test_rows_outside_the_sequences_stay(cuda_device, dtype):
    """Tokens before the first and behind the last sequence hold NaN in every input and are neither used nor written."""
    for D, lens, H in ((64, [90, 39], 4), (128, [90, 39], 4), (40, [90, 39], 4), (64, [129], 3), (128, [901], 3), (64, [777], 4)):
        op, q, k, v, d_o, cu = make(lens, H, H if H == 3 else 2, D, dtype, cuda_device, first=5, tail=70, seed=4)
        end = 5 + sum(lens)
        clean = [x.clone() for x in (q, k, v, d_o)]
        for x in (q, k, v, d_o):
            x[:5] = math.nan
            x[end:] = math.inf
        o, lse = forward(op, q, k, v, cu, fill=3.25)
        for x in (o, lse.t()):
            assert (x[:5] == 3.25).all() and (x[end:] == 3.25).all()
        wo, wl, bo, bl = R.attention_forward(*clean[:3], cu, op.scale, True, dtype)
        within(o[5:end], wo[5:end], bo[5:end], "o")
        within(lse[:, 5:end], wl[:, 5:end], bl[:, 5:end], "lse")
        g = backward(op, q, k, v, o, lse, d_o, cu, fill=1.5)
        want = R.attention_backward(*clean[:3], o, lse, clean[3], cu, op.scale, True, dtype)
        for name, x in g.items():
            assert (x[:5] == 1.5).all() and (x[end:] == 1.5).all(), name
            within(x[5:end], want[name][0][5:end], want[name][1][5:end], name)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, F])
def test_non_finite_values_keep_to_their_sequence(cuda_device, dtype, causal):
    op, q, k, v, d_o, cu = make([100, 60, 77], 2, 1, 64, dtype, cuda_device, causal=causal, seed=5)
    o0, lse0 = forward(op, q, k, v, cu)
    g0 = backward(op, q, k, v, o0, lse0, d_o, cu)
    for x in (q, k, v, d_o):
        x[120] = math.nan
        x[121] = math.inf
        x[122] = -math.inf
    o, lse = forward(op, q, k, v, cu)
    g = backward(op, q, k, v, o, lse, d_o, cu)
    for a, b in [(o, o0), (lse.t(), lse0.t())] + [(g[n], g0[n]) for n in g]:
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[160:], b[160:])
    assert o[120:160].isnan().any()


@pytest.mark.parametrize("lens,H,D", [([150, 90], 2, 64), ([400], 1, 128), ([1500], 16, 128), ([300], 2, 33)], ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_one_value_that_is_not_finite(cuda_device, dtype, lens, H, D):
    """A NaN or infinity in one key alone: the rows that see it have no distribution, or do without the key; the others keep their bits."""
    op, q, k, v, d_o, cu = make(lens, H, H, D, dtype, cuda_device, seed=12)
    clean, _ = forward(op, q, k, v, cu)
    for at in (0, 14, 15, 30, 31, 77, 127, 128, 142):
        for bad in (math.nan, math.inf, -math.inf):
            if at >= lens[0]:
                continue
            k2 = k.clone()
            k2[at, 0, D // 2] = bad
            o, lse = forward(op, q, k2, v, cu)
            s = (q[:lens[0], 0, D // 2].double() * bad)                          # the score's sign, or NaN
            gone = (torch.arange(lens[0], device=cuda_device) >= at) & ~(s == -math.inf)
            gone[0] |= at == 0                                                   # its only key
            assert torch.equal(o[:lens[0], 0].isnan().all(1), gone) and torch.equal(o[:lens[0], 0].isnan().any(1), gone), (at, bad)
            assert torch.equal(lse[0, :lens[0]].isfinite(), ~gone)
            same = torch.ones(o.shape[:2], dtype=torch.bool, device=cuda_device)
            same[at:lens[0], 0] = False
            assert torch.equal(o[same], clean[same]), (at, bad)


@pytest.mark.parametrize("lens,H,D", [([450, 90], 2, 64), ([700], 1, 128), ([700], 40, 64), ([1500], 16, 128), ([700], 2, 33)], ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_tiles_of_keys_at_minus_infinity(cuda_device, dtype, lens, H, D):
    """The first keys have scores of -infinity, tiles of them alone: the same bits as with scores whose exponentials are zero."""
    op, q, k, v, d_o, cu = make(lens, H, H, D, dtype, cuda_device, seed=14)
    q, k = q.clone(), k.clone()
    q[:, :, 1] = 1.0
    for n in (5, 130, 300):
        out = []
        for low in (-3e4, -math.inf):
            k[:n, :, 1] = low
            out.append(forward(op, q, k, v, cu))
        (o0, lse0), (o, lse) = out
        assert not o0.isnan().any() and torch.equal(o[n:], o0[n:]) and torch.equal(lse[:, n:], lse0[:, n:]), n


@pytest.mark.parametrize("lens,H,D", [([150, 90], 2, 64), ([400], 1, 128), ([1500], 16, 128)], ids=str)
@pytest.mark.parametrize("dtype", [BF, F])
def test_values_of_masked_keys_count_for_nothing(cuda_device, dtype, lens, H, D):
    """However large they are: 2^-126 of the type's largest value would already be 4."""
    op, q, k, v, d_o, cu = make(lens, H, H, D, dtype, cuda_device, seed=13)
    o0, lse0 = forward(op, q, k, v, cu)
    dq0 = backward(op, q, k, v, o0, lse0, d_o, cu)["dq"]
    for n in (1, 15, 100, 140):
        v2 = v.clone()
        v2[n:lens[0]] = torch.finfo(dtype).max
        o, lse = forward(op, q, k, v2, cu)
        assert torch.equal(o[:n], o0[:n]) and torch.equal(lse, lse0), n
        assert torch.equal(backward(op, q, k, v2, o, lse, d_o, cu)["dq"][:n], dq0[:n]), n


@pytest.mark.parametrize("dtype", [BF, F])
def test_layouts(cuda_device, dtype):
    """Heads first, a token stride that no 16-byte copy can take, tensors that start between two such boundaries, and key heads
    broadcast over the head dimension."""
    op, q, k, v, d_o, cu = make([70, 130], 4, 2, 64, dtype, cuda_device, seed=6)
    o0, lse0 = forward(op, q, k, v, cu)
    g0 = backward(op, q, k, v, o0, lse0, d_o, cu)
    T = q.shape[0]

    def heads_first(x):
        return x.transpose(0, 1).contiguous().transpose(0, 1)

    def odd(x):
        buf = torch.zeros(T, x.shape[1] * 64 + 3, dtype=dtype, device=cuda_device)
        y = buf[:, 1:1 + x.shape[1] * 64].unflatten(1, (-1, 64))
        y.copy_(x)
        return y
    for lay in (heads_first, odd):
        a = [lay(x) for x in (q, k, v, d_o)]
        o, lse = lay(torch.zeros_like(o0)), torch.zeros_like(lse0)
        op.pm_attention_packed_forward(*a[:3], cu, o, lse)
        wo, wl, bo, bl = R.attention_forward(q, k, v, cu, op.scale, True, dtype)
        within(o, wo, bo, "o")
        within(lse, wl, bl, "lse")
        g = [lay(torch.zeros_like(x)) for x in (q, k, v)]
        op.pm_attention_packed_backward(*a[:3], o, lse, a[3], cu, *g)
        want = R.attention_backward(q, k, v, o, lse, d_o, cu, op.scale, True, dtype)
        for x, (w, b) in zip(g, want.values()):
            within(x, w, b, "gradient")
    one = k[:, :1].expand(-1, 2, -1)
    o, lse = forward(op, q, one, v, cu)
    wo, wl, bo, bl = R.attention_forward(q, one, v, cu, op.scale, True, dtype)
    within(o, wo, bo, "o, broadcast keys")


def test_starts_that_reach_outside(cuda_device):
    """Entries beyond the tensors are clipped; a sequence that would end before it starts is empty."""
    for dtype in (BF, F):
        op, q, k, v, d_o, _ = make([100, 100], 2, 1, 64, dtype, cuda_device, seed=7)
        i32 = dict(dtype=torch.int32, device=cuda_device)
        good = torch.tensor([0, 100, 200], **i32)
        o0, lse0 = forward(op, q, k, v, good)
        g0 = backward(op, q, k, v, o0, lse0, d_o, good)
        for cu in (torch.tensor([-7, 100, 5000], **i32), torch.tensor([-2 ** 31, 100, 2 ** 31 - 1], **i32)):
            o, lse = forward(op, q, k, v, cu)
            assert torch.equal(o, o0) and torch.equal(lse, lse0)
            g = backward(op, q, k, v, o, lse, d_o, cu)
            assert all(torch.equal(g[n], g0[n]) for n in g)
        o, _ = forward(op, q, k, v, torch.tensor([100, 0], **i32), fill=2.0)
        assert (o == 2.0).all()
        o, _ = forward(op, q, k, v, torch.tensor([0], **i32), fill=2.0)
        assert (o == 2.0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_same_bits_every_time_and_without_lse(cuda_device, dtype):
    op, q, k, v, d_o, cu = make([333, 65, 400], 4, 2, 64, dtype, cuda_device, seed=8)
    o, lse = forward(op, q, k, v, cu)
    g = backward(op, q, k, v, o, lse, d_o, cu)
    for _ in range(3):
        o2, lse2 = forward(op, q, k, v, cu)
        g2 = backward(op, q, k, v, o, lse, d_o, cu)
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(g[n], g2[n]) for n in g)
    o3 = torch.zeros_like(o)
    op.pm_attention_packed_forward(q, k, v, cu, o3)
    assert torch.equal(o, o3)


@pytest.mark.parametrize("dtype", [BF, F])
def test_captured_and_on_two_streams(cuda_device, dtype):
    """Two calls at the same time on streams of their own, and a captured forward and backward pass replayed on new inputs."""
    sets = [make([150, 222], 4, 2, 64, dtype, cuda_device, seed=9 + i) for i in range(2)]
    want = []
    for s in sets:
        op, q, k, v, d_o, cu = s
        o, lse = forward(op, q, k, v, cu)
        want.append((o, backward(op, q, k, v, o, lse, d_o, cu)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s, st in zip(sets, streams):
        op, q, k, v, d_o, cu = s
        st.wait_stream(torch.cuda.current_stream())
        o, lse = torch.zeros_like(q), torch.zeros(4, q.shape[0], device=cuda_device)
        g = [torch.zeros_like(x) for x in (q, k, v)]
        st.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            op.pm_attention_packed_forward(q, k, v, cu, o, lse, stream=st)
            op.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, *g, stream=st)
        got.append((o, dict(zip(("dq", "dk", "dv"), g))))
    torch.cuda.synchronize()
    for (o, g), (wo, wg) in zip(got, want):
        assert torch.equal(o, wo) and all(torch.equal(g[n], wg[n]) for n in g)
    op, q, k, v, d_o, cu = [x.clone() if isinstance(x, torch.Tensor) else x for x in sets[0]]
    o, lse = torch.zeros_like(q), torch.zeros(4, q.shape[0], device=cuda_device)
    g = [torch.zeros_like(x) for x in (q, k, v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_attention_packed_forward(q, k, v, cu, o, lse)
        op.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, *g)
    for s, (wo, wg) in reversed(list(zip(sets, want))):
        for x, y in zip((q, k, v, d_o), s[1:5]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, wo) and all(torch.equal(x, wg[n]) for x, n in zip(g, ("dq", "dk", "dv")))
    # other lengths in the captured graph's cu_seqlens: the launch covers any lengths that sum to its tokens
    op2, q2, k2, v2, d2, cu2 = make([1, 371], 4, 2, 64, dtype, cuda_device, seed=20)
    for x, y in zip((q, k, v, d_o, cu), (q2, k2, v2, d2, cu2)):
        x.copy_(y)
    graph.replay()
    wo, _, bo, _ = R.attention_forward(q2, k2, v2, cu2, op2.scale, True, dtype)
    within(o, wo, bo, "o of other lengths")


@pytest.mark.parametrize("D", [64, 33])
def test_offsets_beyond_32_bits(cuda_device, D):
    """Rows 2^25 elements apart: the last of 130 lies 4.3 billion elements behind the first."""
    op, q, k, v, d_o, cu = make([130], 1, 1, D, BF, cuda_device, seed=11)
    far = torch.empty(129 * 2 ** 25 + D, dtype=BF, device=cuda_device).as_strided((130, 1, D), (2 ** 25, D, 1))
    for name in ("q", "k", "v"):
        x = dict(q=q, k=k, v=v)
        far.copy_(x[name])
        x[name] = far
        o, lse = forward(op, **x, cu=cu)
        wo, wl, bo, bl = R.attention_forward(q, k, v, cu, op.scale, True, BF)
        within(o, wo, bo, "o")
    g = [torch.zeros_like(x) for x in (q, k, v)]
    want = R.attention_backward(q, k, v, o, lse, d_o, cu, op.scale, True, BF)
    op.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, g[0], g[1], far)
    within(far, *want["dv"], "dv")
    op.pm_attention_packed_status()


def test_python_refusals(cuda_device):
    import paper_1910_05124_b200 as pm
    op, q, k, v, d_o, cu = make([30, 20], 4, 2, 64, BF, cuda_device)
    o, lse = torch.zeros_like(q), torch.zeros(4, 50, device=cuda_device)
    bad = [dict(q=q.half()), dict(k=k.float()), dict(k=k[:, :1]), dict(v=v[:49]), dict(cu=cu.long()), dict(cu=cu.cpu()), dict(cu=cu[None]),
           dict(o=o.float()), dict(o=o[:1].expand(50, 4, 64)), dict(lse=lse[:, :49]), dict(lse=lse.double()), dict(q=q.transpose(1, 2)),
           dict(q=q[0]), dict(cu=cu[:0])]
    for kw in bad:
        a = dict(q=q, k=k, v=v, cu=cu, o=o, lse=lse)
        a.update(kw)
        with pytest.raises(pm.PipeMareError):
            op.pm_attention_packed_forward(a["q"], a["k"], a["v"], a["cu"], a["o"], a["lse"])
    with pytest.raises(pm.PipeMareError, match="lse"):
        op.pm_attention_packed_backward(q, k, v, o, None, d_o, cu, *[torch.zeros_like(x) for x in (q, k, v)])
    assert (o == 0).all()
