"""The KL term of the policy loss, e^d - d - 1, and its slope e^d - 1, token by token: the first loses its bits for small d."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                    # half a step of fp32
NEAR = np.concatenate([np.linspace(0.5, 1, 60, endpoint=False), [0.49999997, 0.99999994], np.geomspace(1e-6, 0.5, 20)])
FAR = np.concatenate([[1.0, 1.0000001], np.geomspace(1, 30, 20)])


def exact(d):
    """e^d - 1 and e^d - 1 - d of 64-bit numbers; the second by its series below 1, 20 terms of it."""
    term, s = d * d / 2, np.zeros_like(d)
    for n in range(3, 23):
        s, term = s + term, term * d / n
    return np.expm1(d), np.where(np.abs(d) < 1, s, np.expm1(d) - d)


def bounds(d, slope, kl):
    """Near: of the series' sum its FMAs' roundings (1.4 U, as each partial sum is multiplied with d below 1), its constants' (0.6), the terms left
    out (0.1), d^2 and the product with it (2), the result (1): 6 U of kl; the slope is d + kl.  Far: two units in the last place of
    the exponential (4 U), the differences, the result."""
    near = np.abs(d) < 1
    e = 4 * np.exp(d) + np.abs(slope)
    return np.where(near, 6 * kl + 2 * np.abs(slope), e + np.abs(slope)) * U, np.where(near, 6 * kl, e + 2 * kl) * U


@pytest.mark.parametrize("sign", [1, -1])
def test_token_by_token(cuda_device, sign):
    import paper_1910_05124_b200 as pm
    d = torch.tensor(np.concatenate([NEAR, FAR]) * sign, dtype=torch.float32, device=cuda_device)
    zero, stats, grad = torch.zeros_like(d), torch.zeros(5, device=cuda_device), torch.zeros_like(d)
    op = pm.PolicyLoss(kl_coef=1.0, mean=False)
    op.pm_policy_loss(zero, zero, zero, stats, d_logprob=grad, ref_logprob=d)          # log probabilities of 0: d is the reference itself
    kl = torch.zeros(d.numel(), 5, device=cuda_device)
    for i in range(d.numel()):
        op.pm_policy_loss(zero[:1], zero[:1], zero[:1], kl[i], ref_logprob=d[i:i + 1])
    x = d.double().cpu().numpy()
    slope, want = exact(x)
    e_slope, e_kl = bounds(x, slope, want)
    off = np.abs(-grad.double().cpu().numpy() - slope) / e_slope
    assert off.max() <= 1, (x[off.argmax()], off.max())
    off = np.abs(kl[:, 2].double().cpu().numpy() - want) / e_kl
    assert off.max() <= 1, (x[off.argmax()], off.max())


def test_long_lists_alike(cuda_device):
    """The launches of long lists form the same terms."""
    import paper_1910_05124_b200 as pm
    d = torch.linspace(-2, 2, 20000, device=cuda_device)
    zero, op = torch.zeros_like(d), pm.PolicyLoss(kl_coef=1.0, mean=False)
    grads = [torch.zeros_like(d) for _ in range(2)]
    stats = torch.zeros(5, device=cuda_device)
    op.pm_policy_loss(zero, zero, zero, stats, d_logprob=grads[0], ref_logprob=d)
    for at in range(0, 20000, 5000):
        part = slice(at, at + 5000)
        op.pm_policy_loss(zero[part], zero[part], zero[part], stats, d_logprob=grads[1][part], ref_logprob=d[part])
    assert torch.equal(*grads)
