"""The plain forms that the operators are compared with: their gradients against differences of their forward forms, in 64 bits."""
import math

import pytest
import torch

import operators_reference as R


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradient_against_differences(causal):
    gen = torch.Generator().manual_seed(3)
    cu = R.lens_to_cu([3, 0, 1, 4], "cpu", first=1)
    q, k, v, d_o = (torch.randn(11, h, 5, generator=gen, dtype=torch.float64) for h in (4, 2, 2, 4))
    scale = 0.7

    def loss(q, k, v):
        return float((R.attention_forward(q, k, v, cu, scale, causal, torch.float32)[0] * d_o).sum())
    o, lse, _, _ = R.attention_forward(q, k, v, cu, scale, causal, torch.float32)
    got = R.attention_backward(q, k, v, o, lse, d_o, cu, scale, causal, torch.float32)
    h = 1e-5
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        step = torch.randn([q, k, v][at].shape, generator=gen, dtype=torch.float64)
        up, down = ([x + (s * h * step if i == at else 0.0) for i, x in enumerate((q, k, v))] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        # central difference: h^2 times a third derivative of order one, and 2^-52 |loss| / h
        assert abs(slope - float((got[name][0] * step).sum())) < 1e-7, name


def test_logprob_gradient_against_differences():
    gen = torch.Generator().manual_seed(4)
    x = 2 * torch.randn(5, 9, generator=gen, dtype=torch.float64)
    x[1, 3] = -math.inf
    y = torch.tensor([2, 0, -1, 8, 4])
    gl, gh = (torch.randn(5, generator=gen, dtype=torch.float64) for _ in range(2))

    def loss(x):
        out = R.logprobs(x, y, 0)
        return float((out["logprob"] * gl * (y >= 0) + out["entropy"] * gh).sum())
    out = R.logprobs(x, y, 0)
    dx = R.logprobs_backward(x, y, out["lse"], out["entropy"], gl, gh)
    step, h = torch.randn(x.shape, generator=gen, dtype=torch.float64), 1e-5
    slope = (loss(x + h * step) - loss(x - h * step)) / (2 * h)
    assert abs(slope - float((dx * step).sum())) < 1e-7


def test_rows_without_a_distribution():
    x = torch.tensor([[-math.inf] * 3, [0.0, math.nan, 1.0], [0.0, math.inf, 1.0], [1.0, 1.0, -math.inf]])
    out = R.logprobs(x, torch.tensor([0, 0, 1, 1]), 2)
    assert out["lse"][0] == -math.inf and out["entropy"][0] == 0 and out["logprob"][0] == -math.inf
    assert out["lse"][1:3].isnan().all() and (out["top_ids"][1:3] == -1).all()
    assert out["top_ids"][3].tolist() == [0, 1] and abs(float(out["entropy"][3]) - math.log(2)) < 1e-12
