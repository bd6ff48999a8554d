"""The plain 64-bit forms against what they are forms of: published numbers, automatic differentiation, torch's own functions."""
import math

import numpy as np
import torch

import more_operators_reference as M
import operators_reference as R


def test_philox_known_answers():
    """The test vectors published with the generator."""
    got = M.philox([0], 0)[0].tolist()
    assert [f"{x:08x}" for x in got] == ["6627e8d5", "e169c58d", "bc57ac4c", "9b00dbd8"]
    ones = (1 << 128) - 1
    got = M.philox([ones], (1 << 64) - 1)[0].tolist()
    assert [f"{x:08x}" for x in got] == ["408f276d", "41c83b0e", "a20bc7c6", "6d5451fd"]
    # digits of pi: the counter's and the key's words
    counter = sum(x << (32 * i) for i, x in enumerate((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344)))
    got = M.philox([counter], 0xa4093822 | 0x299f31d0 << 32)[0].tolist()
    assert [f"{x:08x}" for x in got] == ["d16cfe09", "94fdcceb", "5001e420", "24126ea1"]


def test_kept_share():
    mask, scale = M.kept(80000, 0.3, 12345, 7)
    assert abs(float(mask.double().mean()) - 0.7) < 0.01 and abs(scale - 1 / 0.7) < 1e-4
    again, _ = M.kept(79992, 0.3, 12345, 8)                  # a counter on: eight elements on
    assert torch.equal(mask[8:], again)


def test_rotation_far_out():
    p = torch.tensor([0, 1, -1, 12345, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    cos, sin = M.rotation(p, 8, 10000.0)
    assert torch.allclose(cos[1], torch.tensor([10000.0 ** (-i / 4) for i in range(4)], dtype=torch.float64).cos())
    assert torch.allclose(sin[2], -sin[1])
    assert abs(float(cos[4, 0]) - math.cos(math.fmod(2 ** 31 - 1, 2 * math.pi))) < 1e-6


def test_norm_gradients():
    gen = torch.Generator().manual_seed(0)
    for inter in (False, True):
        for D, rotary in ((6, 4), (5, 0), (8, 8)):
            x = torch.randn(3, 2, D, generator=gen, dtype=torch.float64).requires_grad_()
            g = torch.randn(D, generator=gen, dtype=torch.float64).requires_grad_()
            d_y = torch.randn(3, 2, D, generator=gen, dtype=torch.float64)
            cos, sin = M.rotation(torch.tensor([0, 3, 100]), rotary, 100.0)
            y = M.norm_forward(x, g, cos, sin, inter, 1e-3, torch.float32)[0]
            want = torch.autograd.grad(y, (x, g), d_y)
            dx, _, dg, _ = M.norm_backward(x.detach(), g.detach(), cos, sin, inter, 1e-3, d_y, torch.float32)
            assert torch.allclose(dx, want[0]) and torch.allclose(dg, want[1])
            if rotary == D:                                  # a rotation keeps lengths, and the norm is the root mean square
                assert torch.allclose(y.square().sum(-1), (x / (x.square().mean(-1, keepdim=True) + 1e-3).sqrt() * g).square().sum(-1))


def test_policy_gradients():
    gen = torch.Generator().manual_seed(1)
    lp = (-torch.rand(50, generator=gen, dtype=torch.float64)).requires_grad_()
    old, adv, ref = lp.detach() + 0.3 * torch.randn(50, generator=gen), torch.randn(50, generator=gen).double(), lp.detach() + torch.randn(50, generator=gen)
    ent, w = torch.rand(50, generator=gen, dtype=torch.float64).requires_grad_(), (torch.rand(50, generator=gen) < 0.7).double()
    ratio = (lp - old).exp()
    share = w / w.sum()
    d = ref - lp
    loss = (share * (-torch.minimum(ratio * adv, ratio.clamp(0.8, 1.3) * adv) + 0.1 * (d.exp() - d - 1) - 0.02 * ent)).sum()
    want = torch.autograd.grad(loss, (lp, ent))
    stats, _, d_lp, _, d_ent = M.policy(lp.detach(), old, adv, ref, ent.detach(), w, 0.2, 0.3, 0.1, 0.02, True)
    assert abs(float(stats[0] - loss.detach())) < 1e-12 and torch.allclose(d_lp, want[0]) and torch.allclose(d_ent, want[1])


def test_cross_gradients():
    gen = torch.Generator().manual_seed(2)
    q, k, v, d_o = (torch.randn(n, h, 4, generator=gen, dtype=torch.float64) for n, h in ((5, 2), (6, 1), (6, 1), (5, 2)))
    cu, cu_kv = R.lens_to_cu([2, 3], "cpu"), R.lens_to_cu([5, 1], "cpu")
    o, lse, _, _ = M.cross_forward(q, k, v, cu, cu_kv, 0.5, torch.float32)
    got = M.cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, 0.5, torch.float32)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    out = torch.zeros_like(q)
    for (a, b), (x, y) in zip(R.spans(cu), R.spans(cu_kv)):
        for h in range(2):
            s = torch.softmax(leaves[0][a:b, h] @ leaves[1][x:y, 0].T * 0.5, 1) @ leaves[2][x:y, 0]
            assert torch.allclose(o[a:b, h], s)
            out = out.index_put((torch.arange(a, b), torch.full((b - a,), h)), s)
    for name, want in zip(("dq", "dk", "dv"), torch.autograd.grad(out, leaves, d_o)):
        assert torch.allclose(got[name][0], want)
    assert np.isfinite(float(lse.sum()))
