"""The policy loss against its 64-bit form, within the bounds that the roundings allow."""
import math

import pytest
import torch

import more_operators_reference as M

pytestmark = pytest.mark.gpu


def make(n, dev, *, seed=0, far=0.3):
    gen = torch.Generator(dev).manual_seed(seed)

    def normal():
        return torch.randn(n, generator=gen, device=dev)
    lp = -4 * torch.rand(n, generator=gen, device=dev)
    return dict(lp=lp, old=lp + far * normal(), adv=normal(), ref=lp + 2 * far * normal(), ent=3 * torch.rand(n, generator=gen, device=dev),
                w=(torch.rand(n, generator=gen, device=dev) < 0.8) * (0.5 + torch.rand(n, generator=gen, device=dev)))


def call(t, low=0.2, high=0.3, kl=0.1, ent=0.02, mean=True, fill=math.nan, grads=True):
    import paper_1910_05124_b200 as pm
    n, dev = t["lp"].numel(), t["lp"].device
    stats, d_lp, d_ent = (torch.full((k,), fill, device=dev) for k in (5, n, n))
    op = pm.PolicyLoss(clip_low=low, clip_high=high, kl_coef=kl, entropy_coef=ent, mean=mean)
    op.pm_policy_loss(t["lp"], t["old"], t["adv"], stats, d_logprob=d_lp if grads else None, ref_logprob=t.get("ref"), entropy=t.get("ent"),
                      d_entropy=d_ent if grads else None, weight=t.get("w"))
    return stats, d_lp, d_ent


def check(t, low=0.2, high=0.3, kl=0.1, ent=0.02, mean=True):
    stats, d_lp, d_ent = call(t, low, high, kl, ent, mean)
    want = M.policy(t["lp"], t["old"], t["adv"], t.get("ref"), t.get("ent"), t.get("w"), low, high, kl, ent, mean)
    for got, w, bound, name in ((stats, want[0], want[1], "stats"), (d_lp, want[2], want[3], "d_logprob"), (d_ent, want[4], 4 * M.U32 * want[4].abs(), "d_entropy")):
        assert not got.isnan().any(), name
        off = (got.double() - w).abs() - bound
        worst = float(off.max()) if off.numel() else 0.0
        assert worst <= 0, f"{name}: {worst} beyond the bound, at {int(off.argmax())}"
    return stats, d_lp, d_ent


# one block, several, a full cluster, the first size of the long lists, many rounds of those
SIZES = [1, 2, 31, 511, 512, 513, 1025, 4095, 4096, 8191, 16383, 16384, 16385, 20000, 303104, 303105, 1000003]


@pytest.mark.parametrize("mean", [True, False])
@pytest.mark.parametrize("n", SIZES)
def test_sizes(cuda_device, n, mean):
    t = make(n, cuda_device, seed=n)
    if not mean:
        t["w"] = t["w"] / n
    check(t, mean=mean)


@pytest.mark.parametrize("n", [300, 20000])
@pytest.mark.parametrize("low,high,kl,ent", [(0.0, 0.0, 0.0, 0.0), (1.0, math.inf, 0.5, 0.0), (0.2, 0.2, 0.0, 0.1), (0.1, 3.0, -0.2, -0.1)])
def test_coefficients(cuda_device, n, low, high, kl, ent):
    t = make(n, cuda_device, seed=1)
    check(t, low, high, kl, ent)
    for without in (("ref",), ("ent",), ("w",), ("ref", "ent", "w")):
        part = {k: v for k, v in t.items() if k not in without}
        check(part, low, high, 0.0 if "ref" in without else kl, 0.0 if "ent" in without else ent)


@pytest.mark.parametrize("n", [300, 20000])
def test_far_and_near(cuda_device, n):
    """Ratios over many orders, and log probabilities that have not moved: the KL term keeps its bits down to zero."""
    check(make(n, cuda_device, seed=2, far=8.0))
    t = make(n, cuda_device, seed=3, far=1e-4)
    check(t)
    t["old"], t["ref"] = t["lp"].clone(), t["lp"].clone()
    stats, d_lp, _ = check(t)
    assert float(stats[2]) == 0 and float(stats[4]) == 0


@pytest.mark.parametrize("n", [300, 20000])
def test_borders(cuda_device, n):
    """Differences that are the borders' nearest floats, on both sides of them: clipped beyond, not before."""
    t = make(n, cuda_device, seed=4)
    t["lp"] = torch.zeros(n, device=cuda_device)
    for border in (math.log1p(0.3), math.log1p(-0.2)):
        x = torch.full((n,), border, device=cuda_device)
        x[1::3], x[2::3] = torch.nextafter(x[1::3], torch.tensor(9.0, device=cuda_device)), torch.nextafter(x[2::3], torch.tensor(-9.0, device=cuda_device))
        t["old"] = -x
        check(t)


@pytest.mark.parametrize("n", [300, 20000])
def test_padding_may_be_anything(cuda_device, n):
    t = make(n, cuda_device, seed=5)
    t["w"][::3] = 0
    clean = check(t)
    dead = t["w"] == 0
    for bad in (math.nan, math.inf, -math.inf):
        for name in ("lp", "old", "adv", "ref", "ent"):
            x = dict(t, **{name: torch.where(dead, bad, t[name])})
            assert all(torch.equal(a, b) for a, b in zip(call(x), clean))
    assert (clean[1][dead] == 0).all() and (clean[2][dead] == 0).all()


@pytest.mark.parametrize("n", [1, 300, 20000])
def test_nothing_counts(cuda_device, n):
    t = make(n, cuda_device, seed=6)
    t["w"] = torch.zeros(n, device=cuda_device)
    for mean in (True, False):
        assert all((x == 0).all() for x in call(t, mean=mean))


def test_no_tokens(cuda_device):
    assert (call(make(0, cuda_device))[0] == 0).all()


@pytest.mark.parametrize("n", [300, 20000])
def test_values_that_are_not_finite(cuda_device, n):
    t = make(n, cuda_device, seed=7)
    t["w"][0] = 1.0
    for name in ("lp", "old", "adv", "ref", "ent"):
        x = dict(t, **{name: t[name].clone()})
        x[name][0] = math.nan
        stats, d_lp, d_ent = call(x)
        assert stats[0].isnan() and not d_lp[1:].isnan().any() and not d_ent[1:].isnan().any()
    x = dict(t, adv=t["adv"].clone(), old=t["old"].clone())
    x["adv"][0], x["old"][0] = 0.0, -math.inf                # an infinite ratio of a token without advantage
    assert not call(x)[0].isnan().any() and not call(x)[1].isnan().any()
    x["adv"][0] = 1.0                                        # clipped
    assert call(x)[0].isfinite().all() and call(x)[1].isfinite().all()
    x["adv"][0] = -1.0
    assert float(call(x)[0][0]) == math.inf
    x = dict(t, w=t["w"].clone())
    x["w"][0] = math.nan
    assert call(x)[0].isnan().any()


@pytest.mark.parametrize("n", [300, 20000])
def test_terms_that_are_measured_alone(cuda_device, n):
    """A term whose coefficient is zero has no part of the loss and the gradient, even where it is infinite."""
    t = make(n, cuda_device, seed=18)
    del t["w"]
    plain = call({k: v for k, v in t.items() if k not in ("ref", "ent")}, kl=0.0, ent=0.0)
    t["ref"], t["ent"] = t["ref"].clone(), t["ent"].clone()
    t["ref"][0], t["ent"][1] = 200.0, math.inf
    stats, d_lp, d_ent = call(t, kl=0.0, ent=0.0)
    assert stats[0] == plain[0][0] and torch.equal(d_lp, plain[1]) and (d_ent == 0).all()
    assert stats[2] == math.inf and stats[3] == math.inf and torch.equal(stats[[1, 4]], plain[0][[1, 4]])


@pytest.mark.parametrize("n", [300, 20000])
def test_statistics_alone(cuda_device, n):
    t = make(n, cuda_device, seed=8)
    want = check(t)[0]
    stats, d_lp, d_ent = call(t, grads=False, fill=7.0)
    assert torch.equal(stats, want) and (d_lp == 7).all() and (d_ent == 7).all()


@pytest.mark.parametrize("n", [300, 16384, 20000, 500000])
def test_captured_replayed_and_repeated(cuda_device, n):
    import paper_1910_05124_b200 as pm
    t = make(n, cuda_device, seed=9)
    stats, d_lp, d_ent = (torch.zeros(k, device=cuda_device) for k in (5, n, n))
    op = pm.PolicyLoss(clip_low=0.2, clip_high=0.3, kl_coef=0.1, entropy_coef=0.02)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            op.pm_policy_loss(t["lp"], t["old"], t["adv"], stats, d_logprob=d_lp, ref_logprob=t["ref"], entropy=t["ent"], d_entropy=d_ent, weight=t["w"])
    for i in range(4):
        for k, v in make(n, cuda_device, seed=10 + i).items():
            t[k].copy_(v)
        for x in (stats, d_lp, d_ent):
            x.fill_(math.nan)
        graphs[i % 2].replay()
        got = [x.clone() for x in (stats, d_lp, d_ent)]
        assert all(torch.equal(a, b) for a, b in zip(got, check(t)))


def test_two_streams(cuda_device):
    t = make(500000, cuda_device, seed=14)
    want = call(t)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append(call(t))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


@pytest.mark.parametrize("n", [40, 20000])
def test_differences(cuda_device, n):
    """Gradients against central differences of the 64-bit form, away from the borders."""
    t = make(n, cuda_device, seed=15)
    stats, d_lp, d_ent = check(t)
    gen = torch.Generator(cuda_device).manual_seed(16)
    way, h = torch.randn(n, generator=gen, device=cuda_device, dtype=torch.float64), 1e-7
    delta = (t["lp"] - t["old"]).double()
    way = torch.where(((delta - math.log1p(0.3)).abs() < 1e-5) | ((delta - math.log1p(-0.2)).abs() < 1e-5), 0.0, way)

    def loss(lp, ent):
        return float(M.policy(lp, t["old"], t["adv"], t["ref"], ent, t["w"], 0.2, 0.3, 0.1, 0.02, True)[0][0])
    lp, ent = t["lp"].double(), t["ent"].double()
    slope = (loss(lp + h * way, ent) - loss(lp - h * way, ent)) / (2 * h)
    assert abs(float((d_lp.double() * way).sum()) - slope) <= 1e-5 * float((d_lp.double() * way).abs().sum()) + 1e-8
    slope = (loss(lp, ent + h * way) - loss(lp, ent - h * way)) / (2 * h)
    assert abs(float((d_ent.double() * way).sum()) - slope) <= 1e-5 * float((d_ent.double() * way).abs().sum()) + 1e-8
