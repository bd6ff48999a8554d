"""Attention over the sequences of another tensor against its 64-bit form, element by element within the bounds that the roundings
allow."""
import math

import pytest
import torch

import more_operators_reference as M
import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def make(lens, kv_lens, H, K, D, dtype, dev, *, first=0, tail=0, seed=0, scale=None, spread=1.0):
    import paper_1910_05124_b200 as pm
    gen = torch.Generator(dev).manual_seed(seed)
    T, S = first + sum(lens) + tail, first + sum(kv_lens) + tail
    q = (spread * torch.randn(T, H, D, generator=gen, device=dev)).to(dtype)
    kv = (spread * torch.randn(S, 2 * K * D, generator=gen, device=dev)).to(dtype)
    k, v = (x.unflatten(1, (-1, D)) for x in kv.split(K * D, 1))
    d_o = torch.randn(T, H, D, generator=gen, device=dev).to(dtype)
    return pm.CrossAttention(H, K, D, scale=scale), q, k, v, d_o, R.lens_to_cu(lens, dev, first), R.lens_to_cu(kv_lens, dev, first)


def forward(op, q, k, v, cu, cu_kv, fill=0.0, **kw):
    o = torch.full(q.shape, fill, dtype=q.dtype, device=q.device)
    lse = torch.full((q.shape[1], q.shape[0]), fill, device=q.device)
    op.pm_attention_cross_forward(q, k, v, cu, cu_kv, o, lse, **kw)
    return o, lse


def backward(op, q, k, v, o, lse, d_o, cu, cu_kv, fill=0.0, **kw):
    # dk and dv in one buffer, as the projection's backward pass wants them
    dq = torch.full(q.shape, fill, dtype=q.dtype, device=q.device)
    buf = torch.full((k.shape[0], 2 * k.shape[1] * k.shape[2]), fill, dtype=q.dtype, device=q.device)
    dk, dv = (x.unflatten(1, (-1, k.shape[2])) for x in buf.split(k.shape[1] * k.shape[2], 1))
    op.pm_attention_cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, dq, dk, dv, **kw)
    return dict(dq=dq, dk=dk, dv=dv)


def within(got, want, bound, what):
    got = got.double()
    assert not got.isnan().any(), what
    same = got == want                                       # infinities among them
    off = torch.where(same, 0.0, (got - want).abs() - bound)
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0, f"{what}: {worst} beyond the bound, at {int(off.argmax())}"


def check(op, q, k, v, d_o, cu, cu_kv, gradients=True):
    o, lse = forward(op, q, k, v, cu, cu_kv)
    wo, wl, bo, bl = M.cross_forward(q, k, v, cu, cu_kv, op.scale, q.dtype)
    within(o, wo, bo, "o")
    within(lse, wl, bl, "lse")
    if gradients:
        got = backward(op, q, k, v, o, lse, d_o, cu, cu_kv)
        for name, (want, bound) in M.cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, op.scale, q.dtype).items():
            within(got[name], want, bound, name)


PAIRS = [([1], [1]), ([1], [300]), ([300], [1]), ([5, 1, 12], [17, 3, 46]), ([64], [65]), ([127, 128, 129], [129, 127, 128]), ([200, 0, 5, 300], [3, 70, 0, 500]),
         ([0, 0], [5, 7]), ([4, 9], [0, 0]), ([256, 255, 257, 1], [100, 475, 256, 640]), ([700, 31], [31, 700]), ([1030], [129])]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens", PAIRS, ids=str)
def test_lengths(cuda_device, lens, kv_lens, dtype):
    check(*make(lens, kv_lens, 2, 1, 64, dtype, cuda_device))
    check(*make(lens, kv_lens, 4, 2, 128, dtype, cuda_device, first=3, tail=9, seed=1))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [1, 7, 8, 24, 32, 33, 56, 64, 72, 80, 96, 120, 128])
def test_head_widths(cuda_device, D, dtype):
    check(*make([130, 70], [50, 200], 2, 2, D, dtype, cuda_device, seed=D))
    check(*make([1, 1, 2], [150, 40, 333], 2, 2, D, dtype, cuda_device, seed=D))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (8, 2), (5, 5), (16, 1), (24, 1)])
def test_shared_heads(cuda_device, H, K, dtype):
    check(*make([40, 150], [220, 33], H, K, 128 if H < 8 else 64, dtype, cuda_device, seed=H))
    check(*make([1, 1], [400, 33], H, K, 64, dtype, cuda_device, seed=H))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens,H,K,D", [
    ([1] * 16, [37 * (i + 1) for i in range(16)], 4, 4, 64), ([1], [5000], 2, 1, 64), ([1, 1, 1], [2, 3001, 0], 8, 2, 128), ([4] * 5, [600, 1, 64, 65, 129], 4, 2, 64),
    ([1, 40, 1, 1, 1, 1, 1, 1, 1], [70] * 9, 2, 2, 64), ([3] * 70, [11 * (i % 9) for i in range(70)], 2, 1, 96), ([1] * 300, [i % 40 for i in range(300)], 1, 1, 64),
    ([16] * 3, [90, 900, 9], 1, 1, 128), ([17] * 3, [90, 900, 9], 2, 2, 80), ([32] * 4, [90, 300, 9, 0], 2, 2, 64), ([8, 9, 3, 0], [90, 300, 9, 5], 8, 2, 128),
    ([5] * 40, [60] * 40, 24, 4, 64), ([1, 60], [700, 300], 4, 2, 48)], ids=str)
def test_few_queries(cuda_device, lens, kv_lens, H, K, D, dtype):
    """Decoding steps: a token or a few to each sequence, one sequence with more among them."""
    check(*make(lens, kv_lens, H, K, D, dtype, cuda_device, first=2, tail=5, seed=len(lens)))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens,H,K,D", [([150], [2000], 2, 1, 64), ([2000], [40], 2, 1, 64), ([90, 3], [1500, 3], 1, 1, 128), ([1, 900], [900, 1], 4, 1, 120),
                                                ([33], [700], 1, 1, 33), ([600], [1300], 1, 1, 64)], ids=str)
def test_few_blocks(cuda_device, lens, kv_lens, H, K, D, dtype):
    """Long sequences and few heads: blocks share the work of one."""
    check(*make(lens, kv_lens, H, K, D, dtype, cuda_device, first=3, tail=50, seed=D))


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_sequences(cuda_device, dtype):
    lens, kv_lens = [(7 * i) % 23 for i in range(300)], [(5 * i) % 31 for i in range(300)]
    check(*make(lens, kv_lens, 2, 1, 32, dtype, cuda_device, seed=1))
    check(*make([130, 257, 64], [64, 130, 300], 40, 8, 64, dtype, cuda_device, seed=2))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens,H,K,D", [
    ([256] * 6, [100, 475, 128, 1, 257, 0], 32, 32, 64), ([130, 257, 64, 0, 300, 33], [64, 130, 300, 40, 0, 700], 64, 16, 48), ([700], [1300], 96, 2, 64),
    ([100] * 40, [(i * 37) % 200 for i in range(40)], 8, 8, 32), ([20] * 200, [20 * (i % 7) for i in range(200)], 48, 48, 64)], ids=str)
def test_more_tiles_than_run_at_a_time(cuda_device, lens, kv_lens, H, K, D, dtype):
    check(*make(lens, kv_lens, H, K, D, dtype, cuda_device, first=2, tail=6, seed=D, spread=2.0), gradients=len(lens) < 100)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens", [[100], [1]])
@pytest.mark.parametrize("spread,scale", [(6.0, None), (0.01, None), (1.0, 2.0)])
def test_peaked_and_flat_scores(cuda_device, dtype, spread, scale, lens):
    check(*make(lens, [400], 2, 1, 64, dtype, cuda_device, spread=spread, scale=scale, seed=2))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens", [[520], [2]])
def test_growing_scores(cuda_device, dtype, lens):
    """Every key tile raises the running maximum by far, so that all sums are rescaled every time; then the reverse."""
    op, q, k, v, d_o, cu, cu_kv = make(lens, [520], 2, 1, 64, dtype, cuda_device, seed=3, scale=0.5)
    ramp = torch.linspace(0.1, 8, 520, device=cuda_device)
    for r in (ramp, ramp.flip(0)):
        check(op, q.abs(), (k.float().abs() * r[:, None, None]).to(dtype), v, d_o, cu, cu_kv)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens,H,K,D", [([90, 39], [39, 150], 4, 2, 64), ([90, 39], [39, 150], 4, 2, 128), ([90, 39], [39, 150], 4, 2, 40), ([129], [777], 3, 3, 64),
                                                ([901], [33], 3, 3, 128), ([1, 1, 1], [33, 130, 200], 4, 2, 64), ([1, 0, 2], [33, 130, 0], 4, 2, 100)], ids=str)
def test_rows_outside_the_sequences_stay(cuda_device, dtype, lens, kv_lens, H, K, D):
    """Rows before the first and behind the last sequence hold NaN and infinities in every input and are neither used nor written."""
    op, q, k, v, d_o, cu, cu_kv = make(lens, kv_lens, H, K, D, dtype, cuda_device, first=5, tail=70, seed=4)
    end, end_kv = 5 + sum(lens), 5 + sum(kv_lens)
    for x, e in ((q, end), (d_o, end), (k, end_kv), (v, end_kv)):
        x[:5] = math.nan
        x[e:] = math.inf
    o, lse = forward(op, q, k, v, cu, cu_kv, fill=3.25)
    g = backward(op, q, k, v, o, lse, d_o, cu, cu_kv, fill=3.25)
    for x, e in ((o, end), (lse.t(), end), (g["dq"], end), (g["dk"], end_kv), (g["dv"], end_kv)):
        assert (x[:5] == 3.25).all() and (x[e:] == 3.25).all()
    inside, inside_kv = slice(5, end), slice(5, end_kv)
    q2, d2, k2, v2 = q.clone(), d_o.clone(), k.clone(), v.clone()
    for x, e in ((q2, end), (d2, end), (k2, end_kv), (v2, end_kv)):
        x[:5] = 0
        x[e:] = 0
    wo, wl, bo, bl = M.cross_forward(q2, k2, v2, cu, cu_kv, op.scale, dtype)
    within(o[inside], wo[inside], bo[inside], "o")
    within(lse[:, inside], wl[:, inside], bl[:, inside], "lse")
    o2, lse2 = o.clone(), lse.clone()
    want = M.cross_backward(q2, k2, v2, o2, lse2, d2, cu, cu_kv, op.scale, dtype)
    for name, rows in (("dq", inside), ("dk", inside_kv), ("dv", inside_kv)):
        within(g[name][rows], want[name][0][rows], want[name][1][rows], name)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens", [[70, 20, 65], [1, 1, 1]])
@pytest.mark.parametrize("D", [64, 128, 36])
def test_values_that_are_not_finite_stay_in_their_sequence(cuda_device, dtype, D, lens):
    op, q, k, v, d_o, cu, cu_kv = make(lens, [150, 37, 100], 4, 2, D, dtype, cuda_device, seed=5)
    clean = forward(op, q, k, v, cu, cu_kv)
    clean_g = backward(op, q, k, v, *clean, d_o, cu, cu_kv)
    for x, row in ((v, 160), (k, 160), (v, 186)):            # of the second sequence
        bad = x.clone()
        bad[row] = math.nan
        args = [bad if y is x else y for y in (q, k, v)]
        o, lse = forward(op, *args, cu, cu_kv)
        g = backward(op, *args, o, lse, d_o, cu, cu_kv)
        a, b = lens[0], lens[0] + lens[1]
        assert o[a:b, :].isnan().any(-1).all()
        for got, want, lo, hi in ((o, clean[0], a, b), (lse.t(), clean[1].t(), a, b), (g["dq"], clean_g["dq"], a, b), (g["dk"], clean_g["dk"], 150, 187),
                                  (g["dv"], clean_g["dv"], 150, 187)):
            assert torch.equal(got[:lo], want[:lo]) and torch.equal(got[hi:], want[hi:])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens", [[40, 3], [1, 1]])
def test_scores_of_minus_infinity(cuda_device, dtype, lens):
    """Keys whose score is -infinity count for nothing; a row of nothing else has lse -infinity."""
    op, q, k, v, d_o, cu, cu_kv = make(lens, [200, 150], 2, 1, 64, dtype, cuda_device, seed=6)
    q = q.abs() + 0.1
    k = k.clone()
    k[20:150] = -math.inf
    o, lse = forward(op, q, k, v, cu, cu_kv)
    keep = torch.tensor([i for i in range(350) if not 20 <= i < 150], device=cuda_device)
    wo, wl, bo, bl = M.cross_forward(q, k[keep], v[keep], cu, R.lens_to_cu([70, 150], cuda_device), op.scale, dtype)
    within(o, wo, bo, "o")
    within(lse, wl, bl, "lse")
    k[:200] = -math.inf
    o, lse = forward(op, q, k, v, cu, cu_kv)
    assert (lse[:, :lens[0]] == -math.inf).all() and o[:lens[0]].isnan().all() and not o[lens[0]:].isnan().any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens", [([70, 130], [300, 20]), ([1, 2], [300, 20])])
def test_strides(cuda_device, dtype, lens, kv_lens):
    """Heads before tokens, rows of odd lengths, and views that no 16-byte copy can take give the same results."""
    H, K, D = 4, 2, 64
    op, q, k, v, d_o, cu, cu_kv = make(lens, kv_lens, H, K, D, dtype, cuda_device, seed=7)
    want = M.cross_forward(q, k, v, cu, cu_kv, op.scale, dtype)

    def layouts(x):
        n, h, d = x.shape
        yield x.transpose(0, 1).contiguous().transpose(0, 1)                   # [heads, tokens, d] in memory
        wide = torch.zeros(n, h, d + 8, dtype=x.dtype, device=x.device)[:, :, :d]
        yield wide.copy_(x)
        odd = torch.zeros(n * h * d + 1 + n, dtype=x.dtype, device=x.device)[1:].as_strided((n, h, d), (h * d + 1, d, 1), 1)
        yield odd.copy_(x)
    for ql, kl, vl, ol in zip(*(layouts(x) for x in (q, k, v, torch.zeros_like(q)))):
        lse = torch.zeros(H, q.shape[0], device=cuda_device)
        op.pm_attention_cross_forward(ql, kl, vl, cu, cu_kv, ol, lse)
        within(ol, want[0], want[2], "o")
        within(lse, want[1], want[3], "lse")
        g = [torch.zeros_like(x) for x in (q, k, v)]
        op.pm_attention_cross_backward(ql, kl, vl, ol, lse, d_o, cu, cu_kv, *g)
        back = M.cross_backward(ql, kl, vl, ol, lse, d_o, cu, cu_kv, op.scale, dtype)
        for x, name in zip(g, ("dq", "dk", "dv")):
            within(x, *back[name], name)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens,H,K,D", [([1, 2], [300, 40], 4, 2, 64), ([100, 30], [50, 400], 4, 2, 128), ([700, 300, 0, 4], [200, 100, 5, 0], 64, 64, 64), ([60], [90], 3, 1, 33)], ids=str)
def test_without_lse_on_another_stream(cuda_device, lens, kv_lens, H, K, D, dtype):
    """An evaluation needs no statistics; the call goes to the stream that is given."""
    op, q, k, v, _, cu, cu_kv = make(lens, kv_lens, H, K, D, dtype, cuda_device, seed=17)
    want, _ = forward(op, q, k, v, cu, cu_kv)
    o, stream = torch.zeros_like(q), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    op.pm_attention_cross_forward(q, k, v, cu, cu_kv, o, stream=stream)
    stream.synchronize()
    assert torch.equal(o, want)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,H,K,D", [([3, 5], 2, 1, 64), ([200, 90], 4, 2, 128), ([70] * 12, 48, 48, 64), ([9] * 300, 2, 1, 32)], ids=str)
def test_starts_out_of_range(cuda_device, lens, H, K, D, dtype):
    """Starts before the first and behind the last row are clipped to the tensors, on either side."""
    op, q, k, v, d_o, cu, cu_kv = make(lens, [2 * n for n in lens], H, K, D, dtype, cuda_device, seed=18)
    far, far_kv = cu.clone(), cu_kv.clone()
    far[0], far[-1], far_kv[0], far_kv[-1] = -7, q.shape[0] + 1000, -2 ** 31, 2 ** 31 - 1
    o, lse = forward(op, q, k, v, cu, cu_kv)
    o2, lse2 = forward(op, q, k, v, far, far_kv)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    a, b = backward(op, q, k, v, o, lse, d_o, cu, cu_kv), backward(op, q, k, v, o, lse, d_o, far, far_kv)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", [BF, F])
def test_no_rows_on_one_side(cuda_device, dtype):
    op, q, k, v, d_o, cu, cu_kv = make([3, 4], [5, 6], 2, 1, 64, dtype, cuda_device, first=1, tail=2)
    none, none_q = k[:0], q[:0]
    empty = torch.zeros(3, dtype=torch.int32, device=cuda_device)
    o, lse = forward(op, q, none, none, cu, empty, fill=7.0)
    assert (o[1:8] == 0).all() and (lse[:, 1:8] == -math.inf).all() and (o[:1] == 7).all() and (o[8:] == 7).all() and (lse[:, 8:] == 7).all()
    g = backward(op, q, none, none, o, lse, d_o, cu, empty, fill=7.0)
    assert (g["dq"][1:8] == 0).all() and (g["dq"][8:] == 7).all()
    o, lse = forward(op, none_q, k, v, empty, cu_kv)
    g = backward(op, none_q, k, v, o, lse, d_o[:0], empty, cu_kv, fill=7.0)
    for x in (g["dk"], g["dv"]):
        assert (x[:1] == 7).all() and (x[1:12] == 0).all() and (x[12:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [64, 128, 36])
def test_differences(cuda_device, dtype, D):
    """The gradients of a linear function of o against central differences of the 64-bit form, which the bounds above lean on."""
    op, q, k, v, d_o, cu, cu_kv = make([5, 2], [7, 3], 2, 1, D, dtype, cuda_device, seed=8)
    o, lse = forward(op, q, k, v, cu, cu_kv)
    g = backward(op, q, k, v, o, lse, d_o, cu, cu_kv)
    gen = torch.Generator(cuda_device).manual_seed(9)
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [t.double() for t in (q, k, v)]
        way, h = torch.randn(x[i].shape, generator=gen, device=cuda_device, dtype=torch.float64), 1e-6
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * way, x[i] - h * way
        slope = sum(s * float((M.cross_forward(*y, cu, cu_kv, op.scale, F)[0] * d_o.double()).sum()) for s, y in ((1, up), (-1, down))) / (2 * h)
        want = M.cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, op.scale, dtype)[name]
        # the kernel's bound in this direction, what o's and lse's roundings move (delta by up to |d_o . o| u), and the differences' own 1e-6
        slack = float((want[1] * way.abs()).sum()) + 1e-6 * (1 + abs(slope)) + 4 * R.u(dtype) * float((g[name].double().abs() * way.abs()).sum())
        slack += 2 * R.u(dtype) * op.scale * float((d_o.double() * o.double()).abs().sum()) * float(x[1 - i].abs().max() * way.abs().max()) if i < 2 else 0.0
        assert abs(float((g[name].double() * way).sum()) - slope) <= slack


@pytest.mark.parametrize("dtype", [BF, F])
def test_same_bits_every_time(cuda_device, dtype):
    for lens, kv_lens in (([1] * 6, [900, 20, 333, 64, 1, 70]), ([150, 40], [600, 1100])):
        op, q, k, v, d_o, cu, cu_kv = make(lens, kv_lens, 4, 2, 64, dtype, cuda_device, seed=10)
        first = None
        for _ in range(5):
            o, lse = forward(op, q, k, v, cu, cu_kv)
            now = (o, lse, *backward(op, q, k, v, o, lse, d_o, cu, cu_kv).values())
            assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
            first = now


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lens,kv_lens", [([1] * 4, [300, 5, 80, 40]), ([100, 30], [300, 125])])
def test_captured_and_replayed_with_other_lengths(cuda_device, dtype, lens, kv_lens):
    """Both arrays are read on the device: results of a replayed graph are those of the new lengths."""
    op, q, k, v, d_o, cu, cu_kv = make(lens, kv_lens, 4, 2, 64, dtype, cuda_device, seed=11)
    k, v = k.clone(), v.clone()
    o, lse = torch.zeros_like(q), torch.zeros(4, q.shape[0], device=cuda_device)
    g = [torch.zeros_like(x) for x in (q, k, v)]
    op.pm_attention_cross_forward(q, k, v, cu, cu_kv, o, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_attention_cross_forward(q, k, v, cu, cu_kv, o, lse)
        op.pm_attention_cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, *g)
    n, total, total_kv = len(lens), sum(lens), sum(kv_lens)
    for i, (a, b) in enumerate((([total] + [0] * (n - 1), [1] * (n - 1) + [total_kv - n + 1]), ([0] * (n - 1) + [total], [0] * (n - 1) + [total_kv]),
                                (lens[::-1], kv_lens))):
        new = make(a, b, 4, 2, 64, dtype, cuda_device, seed=12 + i)[1:]
        for x, y in zip((q, k, v, d_o, cu, cu_kv), new):
            x.copy_(y)
        for x in (o, lse, *g):
            x.fill_(math.nan)
        graph.replay()
        wo, wl, bo, bl = M.cross_forward(q, k, v, cu, cu_kv, op.scale, dtype)
        within(o, wo, bo, f"o of {a}, {b}")
        within(lse, wl, bl, f"lse of {a}, {b}")
        want = M.cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, op.scale, dtype)
        for x, name in zip(g, want):
            within(x, *want[name], f"{name} of {a}, {b}")


def test_two_streams(cuda_device):
    """Calls on two streams at the same time, each with a workspace of its own."""
    op, q, k, v, d_o, cu, cu_kv = make([150, 40], [600, 1100], 4, 2, 64, BF, cuda_device, seed=15)
    o, lse = forward(op, q, k, v, cu, cu_kv)
    want = backward(op, q, k, v, o, lse, d_o, cu, cu_kv)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append(backward(op, q, k, v, o, lse, d_o, cu, cu_kv))
    torch.cuda.synchronize()
    assert all(torch.equal(g[n], want[n]) for g in got for n in want)


@pytest.mark.parametrize("dtype", [BF, F])
def test_offsets_beyond_32_bits(cuda_device, dtype):
    """Keys whose rows lie more than 2^32 elements apart."""
    D, K, rows = 64, 1, 70000
    if torch.cuda.get_device_properties(cuda_device).total_memory < 60 << 30:
        pytest.skip("needs 60 GB")
    stride = (1 << 32) // rows + 64
    stride -= stride % 64
    big = torch.zeros(rows * stride, dtype=BF, device=cuda_device) if dtype == BF else torch.zeros(rows * stride, dtype=F, device=cuda_device)
    assert big.numel() > 1 << 32
    op, q, k, v, d_o, cu, cu_kv = make([1, 3], [rows - 150, 150], 2, K, D, dtype, cuda_device, seed=16)
    far = big.as_strided((rows, K, D), (stride, D, 1))
    far.copy_(k)
    a, b = forward(op, q, k, v, cu, cu_kv), forward(op, q, far, v, cu, cu_kv)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    o, lse = a
    g = backward(op, q, k, v, o, lse, d_o, cu, cu_kv)
    dq, dv = torch.zeros_like(q), torch.zeros(rows, K, D, dtype=dtype, device=cuda_device)
    op.pm_attention_cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, dq, far, dv)
    assert torch.equal(far, g["dk"]) and torch.equal(dq, g["dq"]) and torch.equal(dv, g["dv"])
