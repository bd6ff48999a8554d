"""Token log probabilities, entropy, top alternatives and their gradient against the 64-bit forms."""
import math

import pytest
import torch

import operators_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def forward(logits, targets, k, vocab=None):
    import paper_1910_05124_b200 as pm
    n, dev = logits.shape[0], logits.device
    out = {name: torch.full((n,), 7.0, device=dev) for name in ("logprob", "entropy", "lse")}
    out["top_logprob"] = torch.full((n, k), 7.0, device=dev) if k else None
    out["top_ids"] = torch.full((n, k), -7, dtype=torch.int32, device=dev) if k else None
    pm.TokenLogProbs(vocab or logits.shape[1], top_k=k).pm_token_logprobs(logits, targets, **out)
    return {name: x for name, x in out.items() if x is not None}


def bounds(x):
    """Largest error of lse, log probabilities and entropy for finite rows x: the sum of v terms, an exponential (2^-21), the
    logarithm, differences of numbers up to the spread of the row, lse's own rounding, and for the entropy the quotient."""
    f = x[x.isfinite()].double()
    big = float(f.abs().max()) if f.numel() else 0.0
    spread = 2 * big + 20
    # a thread adds at most vocab / 256 terms (all of a short row), then trees
    sums = (x.shape[1] / 256 + 64) * R.SUM + 2.0 ** -21 + 4 * R.SUM * 20
    lse = sums + 4 * R.SUM * (big + 20)
    return dict(lse=lse, logprob=lse + 4 * R.SUM * spread, top_logprob=lse + 4 * R.SUM * spread, entropy=2 * sums * 20 + 8 * R.SUM * 20)


def check(logits, targets, k):
    got, want, b = forward(logits, targets, k), R.logprobs(logits, targets, k), bounds(logits)
    for name, x in got.items():
        w = want[name]
        if name == "top_ids":
            assert torch.equal(x, w)
            continue
        fine = w.isfinite()
        assert torch.equal(x.isnan(), w.isnan()) and torch.equal(x[~fine & ~w.isnan()].double(), w[~fine & ~w.isnan()]), name
        off = (x.double() - w)[fine].abs()
        assert off.numel() == 0 or float(off.max()) <= b[name], (name, float(off.max()), b[name])
    return got


def check_backward(logits, targets, got, gl, gh, in_place=False):
    import paper_1910_05124_b200 as pm
    x = logits.clone() if in_place else logits
    dx = x if in_place else torch.full_like(logits, 7.0)
    want = R.logprobs_backward(logits, targets, got["lse"], got["entropy"], gl, gh)
    pm.TokenLogProbs(logits.shape[1]).pm_token_logprobs_backward(x, targets, got["lse"], dx, d_logprob=gl, entropy=got["entropy"], d_entropy=gh)
    assert torch.equal(dx.isnan(), want.isnan())
    fine = ~want.isnan()
    # p: the difference with lse, its product with log2(e), the exponential; then two or three operations on terms of size
    # |g_l| + |g_H| (|log p| + H), times p; one at the target; the rounding of the result
    logp = (logits.double() - got["lse"].double()[:, None]).clamp(min=-200.0, max=0.0).nan_to_num(neginf=-200.0)
    coarse = (got["lse"].abs() > 4096)[:, None] & got["lse"].isfinite()[:, None]
    logp = torch.where(coarse, torch.log_softmax(torch.where(coarse, logits.double(), 0.0), 1).clamp(min=-200.0), logp)
    p = logp.exp()
    size = torch.zeros_like(p)
    if gl is not None:
        size += gl.double().abs()[:, None]
    if gh is not None:
        size += gh.double().abs()[:, None] * (logp.abs() + got["entropy"].double().abs()[:, None].nan_to_num())
    # the absolute error of log p is the rounding of the difference: at most that of |x| + |lse|
    far = (logits.double().abs().nan_to_num(posinf=0.0) + got["lse"].double().abs()[:, None].nan_to_num(posinf=0.0)).clamp(max=1e4)
    far = torch.where(coarse, 300.0, far)                     # ... which rows of a large lse do not take
    rel = 4 * R.SUM * (far + logp.abs()) + 2.0 ** -21
    bound = p * size * (rel + 8 * R.SUM) + p * (4 * R.SUM * far) * (gh.double().abs()[:, None] if gh is not None else 0.0)
    if gl is not None:
        bound = bound + 2 * R.SUM * gl.double().abs().nan_to_num()[:, None]
    bound = bound + R.u(logits.dtype) * want.abs() + 2.0 ** -126          # results below the normal range may be flushed
    off = ((dx.double() - want).abs() - bound)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())


def make(n, v, dtype, dev, seed=0, spread=3.0):
    gen = torch.Generator(dev).manual_seed(seed)
    x = (spread * torch.randn(n, v, generator=gen, device=dev)).to(dtype)
    y = torch.randint(0, v, (n,), generator=gen, device=dev).to(torch.int32)
    gl, gh = (torch.randn(n, generator=gen, device=dev) for _ in range(2))
    return x, y, gl, gh


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("n,v,k", [(1, 1, 1), (3, 2, 2), (5, 31, 4), (2, 32, 32), (7, 1000, 8), (9, 1023, 20), (3, 1024, 0), (5, 1025, 7), (9, 2047, 20), (5, 2049, 7), (1024, 4096, 6),
                                   (1100, 3999, 20), (4, 4097, 1), (1, 32000, 8), (3, 50001, 20),
                                   (33, 8191, 5), (150, 8192, 0), (300, 12345, 3), (1, 131071, 32)])
def test_sizes(cuda_device, n, v, k, dtype):
    x, y, gl, gh = make(n, v, dtype, cuda_device, seed=v)
    y[0] = -1 if n > 1 else y[0]
    got = check(x, y, k)
    check_backward(x, y, got, gl, gh)
    check_backward(x, y, got, gl, None, in_place=True)
    check_backward(x, None, got, None, gh)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("v,k", [(40, 5), (900, 32), (1024, 3), (1501, 32), (3001, 8), (20000, 8), (20000, 32)])
def test_ties_go_to_the_lowest_id(cuda_device, dtype, v, k):
    """Few distinct values, one value, sorted rows, the best next to each other, signed zeros."""
    gen = torch.Generator(cuda_device).manual_seed(v)
    rows = [torch.randint(0, 3, (v,), generator=gen, device=cuda_device).float(), torch.zeros(v, device=cuda_device),
            torch.arange(v, device=cuda_device) / v, -torch.arange(v, device=cuda_device) / v, torch.zeros(v, device=cuda_device),
            -torch.zeros(v, device=cuda_device)]
    rows[4][v // 2:v // 2 + k + 1] = 5.0
    rows[5][v // 3] = 0.0
    check(torch.stack(rows).to(dtype), None_targets(len(rows), cuda_device), k)


def None_targets(n, dev):
    return torch.zeros(n, dtype=torch.int32, device=dev)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("v", [33, 5000, 40000])
def test_infinities_and_nan(cuda_device, dtype, v):
    x, y, gl, gh = make(9, v, dtype, cuda_device, seed=v)
    x[0] = -math.inf                                         # nothing left
    x[1, v // 2] = math.nan
    x[2, v - 1] = math.inf
    x[3, 1:] = -math.inf                                     # one token left
    x[4, ::2] = -math.inf
    x[5] = torch.finfo(dtype).min                            # the lowest value everywhere
    x[6] = torch.finfo(dtype).min
    x[6, 7] = 2.0
    x[7] = torch.finfo(dtype).max
    x[7, 3] = torch.finfo(dtype).min
    y[0], y[3], y[4], y[6], y[7], y[8] = 3, 5, 2, 7, 3, v    # masked targets, and one beyond the vocabulary
    got = forward(x, y, 6)
    want = R.logprobs(x, y, 6)
    assert torch.equal(got["top_ids"], want["top_ids"])
    b = bounds(x[8:])
    for name in ("logprob", "entropy", "lse", "top_logprob"):
        g, w = got[name].double(), want[name]
        w = torch.where(w.abs() > 3.4028235677973366e38, w.sign() * math.inf, w)      # a log probability below fp32's range
        assert torch.equal(g.isnan(), w.isnan()), name
        assert torch.equal(g.isinf(), w.isinf()) and torch.equal(g[g.isinf()], w[w.isinf()]), name
        fine = w.isfinite()
        assert ((g - w)[fine].abs() <= b[name] + 2.0 ** -23 * w[fine].abs()).all(), name
    check_backward(x, y, got, gl, gh)
    check_backward(x, y, got, gl, None, in_place=True)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("v", [3, 33, 5000, 40000])
def test_masked_rows_far_from_zero(cuda_device, dtype, v):
    """Tokens at -infinity beside logits whose logsumexp lies beyond 4096: they have no part of the sum."""
    x, y, gl, gh = make(8, v, dtype, cuda_device, seed=v + 1)
    for row, (far, every) in enumerate([(6000.0, 2), (-6000.0, 2), (1e30, 3), (-1e30, 3), (4200.0, 1), (torch.finfo(dtype).min, 2), (torch.finfo(dtype).max, 2)]):
        x[row] = (x[row].float() + far).clamp(min=torch.finfo(dtype).min, max=torch.finfo(dtype).max).to(dtype)
        x[row, 1::every] = -math.inf
        y[row] = 0 if row % 2 else 1
    got = forward(x, y, 2)
    want = R.logprobs(x, y, 2)
    b = bounds(x[7:])
    for name in ("entropy", "lse"):
        assert ((got[name].double() - want[name]).abs() <= b[name] + 2.0 ** -23 * want[name].abs()).all(), name
    check_backward(x, y, got, gl, gh)
    check_backward(x, y, got, gl, None, in_place=True)


@pytest.mark.parametrize("dtype", [F, BF])
def test_strides_and_alignment(cuda_device, dtype):
    """Rows of a wider tensor that start at every place within 16 bytes; gradients with the same and with other strides."""
    import paper_1910_05124_b200 as pm
    for first in range(0, 9, 2):
        for v in (257, 6000):
            base, y, gl, gh = make(6, v + 11, dtype, cuda_device, seed=first)
            y.clamp_(max=v - 1)
            x = base[:, first:first + v]
            keep = base.clone()
            got, want = forward(x, y, 4, vocab=v), forward(x.contiguous(), y, 4)
            for n in got:
                same = torch.equal(got[n], want[n]) if n == "top_ids" else torch.allclose(got[n], want[n], rtol=0, atol=2 * bounds(x)[n])
                assert same, n
            assert torch.equal(base, keep)
            op = pm.TokenLogProbs(v)
            ref = torch.zeros(6, v, dtype=dtype, device=cuda_device)
            op.pm_token_logprobs_backward(x.contiguous(), y, got["lse"], ref, d_logprob=gl, entropy=got["entropy"], d_entropy=gh)
            for width, at in ((v + 11, first), (v + 3, 1), (v, 0)):
                buf = torch.full((6, width), 9.0, dtype=dtype, device=cuda_device)
                dx = buf[:, at:at + v]
                op.pm_token_logprobs_backward(x, y, got["lse"], dx, d_logprob=gl, entropy=got["entropy"], d_entropy=gh)
                assert torch.equal(dx, ref)
                assert (buf[:, :at] == 9.0).all() and (buf[:, at + v:] == 9.0).all()


def test_offsets_beyond_32_bits(cuda_device):
    """Rows 2^28 elements apart, 20 of them, within one tensor."""
    import paper_1910_05124_b200 as pm
    x, y, gl, gh = make(20, 700, BF, cuda_device, seed=3)
    far = torch.empty(19 * 2 ** 28 + 700, dtype=BF, device=cuda_device).as_strided((20, 700), (2 ** 28, 1))
    far.copy_(x)
    got = check(far, y, 4)
    op, ref = pm.TokenLogProbs(700), torch.zeros_like(x)
    op.pm_token_logprobs_backward(x, y, got["lse"], ref, d_logprob=gl)
    op.pm_token_logprobs_backward(far, y, got["lse"], far, d_logprob=gl)
    assert torch.equal(far, ref)


def test_optional_results_streams_and_graphs(cuda_device):
    import paper_1910_05124_b200 as pm
    x, y, gl, gh = make(20, 3000, F, cuda_device)
    full = forward(x, y, 3)
    op = pm.TokenLogProbs(3000)
    lp = torch.zeros(20, device=cuda_device)
    op.pm_token_logprobs(x, y, lp)
    assert torch.equal(lp, full["logprob"])
    lse = torch.zeros(20, device=cuda_device)
    op.pm_token_logprobs(x, None, None, lse=lse)
    assert torch.equal(lse, full["lse"])
    op.pm_token_logprobs(x[:0], y[:0], lp[:0])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(20, device=cuda_device)
    dx = torch.zeros_like(x)
    st.wait_stream(torch.cuda.current_stream())
    op.pm_token_logprobs(x, y, out, lse=lse, stream=st)
    op.pm_token_logprobs_backward(x, y, lse, dx, d_logprob=gl, stream=st)
    st.synchronize()
    assert torch.equal(out, full["logprob"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.pm_token_logprobs(x, y, lp, lse=lse)
        op.pm_token_logprobs_backward(x, y, lse, dx, d_logprob=gl)
    x2, y2, _, _ = make(20, 3000, F, cuda_device, seed=5)
    x.copy_(x2)
    y.copy_(y2)
    graph.replay()
    want = forward(x2, y2, 0)
    ref = torch.zeros_like(x)
    op.pm_token_logprobs_backward(x2, y2, want["lse"], ref, d_logprob=gl)
    assert torch.equal(lp, want["logprob"]) and torch.equal(dx, ref)


def test_python_refusals(cuda_device):
    import paper_1910_05124_b200 as pm
    x, y, gl, gh = make(4, 50, F, cuda_device)
    op, lp = pm.TokenLogProbs(50, top_k=2), torch.zeros(4, device=cuda_device)
    top = dict(top_logprob=torch.zeros(4, 2, device=cuda_device), top_ids=torch.zeros(4, 2, dtype=torch.int32, device=cuda_device))
    for a in ((x.double(), y, lp), (x[:, :49], y, lp), (x.t().contiguous().t(), y, lp), (x, y.long(), lp), (x, y.cpu(), lp), (x, y[:3], lp),
              (x, y, lp.double()), (x, y, None), (x, None, lp), (x[:1].expand(4, 50), y, lp), (x[0], y, lp)):
        with pytest.raises(pm.PipeMareError):
            op.pm_token_logprobs(*a, **top)
    with pytest.raises(pm.PipeMareError, match="top"):
        op.pm_token_logprobs(x, y, lp)
    dx = torch.zeros_like(x)
    for a, kw in (((x, y, lp, dx), {}), ((x, None, lp, dx), dict(d_logprob=gl)), ((x, y, lp, dx), dict(d_entropy=gh)), ((x, y, None, dx), dict(d_logprob=gl)),
                  ((x, y, lp, dx.bfloat16()), dict(d_logprob=gl)), ((x, y, lp, dx[:3]), dict(d_logprob=gl))):
        with pytest.raises(pm.PipeMareError):
            op.pm_token_logprobs_backward(*a, **kw)
    assert (lp == 0).all() and (dx == 0).all()
