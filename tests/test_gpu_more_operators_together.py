"""The operators as a program uses them: one step of policy-gradient training of a small encoder-decoder's decoder, from its embedded
tokens and the encoder's states to the clipped gradients, against the same step in 64 bits; then a decoding step of the same weights."""
import pytest
import torch

import more_operators_reference as M
import operators_reference as R

pytestmark = pytest.mark.gpu


def attend(q, k, v, cu, cu_kv, scale, causal):
    """Differentiable attention in 64 bits; rows outside the sequences are zero."""
    group, out = q.shape[1] // k.shape[1], []
    at = 0
    for (a, b), (x, y) in zip(R.spans(cu), R.spans(cu_kv)):
        heads = []
        for i in range(q.shape[1]):
            s = (q[a:b, i] @ k[x:y, i // group].T) * scale
            if causal:
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
            heads.append(torch.softmax(s, 1) @ v[x:y, i // group])
        out.append(torch.stack(heads, 1))
        at = b
    return torch.cat(out + [torch.zeros(q.shape[0] - at, *q.shape[1:], dtype=q.dtype, device=q.device)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_policy_gradient_step_and_decoding(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    dev = cuda_device
    gen = torch.Generator(dev).manual_seed(3)
    f32 = dict(dtype=torch.float32, device=dev)
    H, K, D, vocab, width, p = 4, 2, 64, 520, 128, 0.25
    lens, kv_lens, tail = [37, 1, 90], [50, 130, 7], 6
    n, T, S = sum(lens), sum(lens) + tail, sum(kv_lens)
    cu, cu_kv = R.lens_to_cu(lens, dev), R.lens_to_cu(kv_lens, dev)
    positions = torch.cat([torch.arange(x, device=dev) for x in lens + [tail]]).to(torch.int32)
    # projections of the tokens, output, queries of the cross attention, projections of the states, output, vocabulary; four gains
    shapes = [((H + 2 * K) * D, width), (width, H * D), (H * D, width), (2 * K * D, width), (width, H * D), (vocab, width), (D,), (D,), (D,), (D,)]
    sizes = [s[0] * (s[1] if len(s) > 1 else 1) for s in shapes]
    starts = [sum(sizes[:i]) for i in range(len(sizes))]
    total = sum(sizes)
    w = torch.randn(total, generator=gen, device=dev) * width ** -0.5
    w[starts[6]:] = 1 + 0.1 * torch.randn(4 * D, generator=gen, device=dev)

    def split(flat):
        return [flat[a:a + k].view(s) for a, k, s in zip(starts, sizes, shapes)]
    x, e = (torch.randn(k, width, generator=gen, device=dev).to(dtype) for k in (T, S))
    y = torch.randint(0, vocab, (T,), generator=gen, device=dev).to(torch.int32)
    rng = torch.tensor([77, 1000], dtype=torch.int64, device=dev)
    masks = [M.kept(T * width, p, 77, 1000 + i * pm.Dropout.counters(T * width)) for i in range(2)]

    # the step in 64 bits, of the rounded weights
    leaf = w.double().requires_grad_()
    mats = split(leaf)
    if dtype != torch.float32:
        mats = [m + (m.detach().to(dtype).double() - m.detach()) if m.dim() == 2 else m for m in mats]
    wqkv, wo, wq2, wkv, wo2, wv, *g = mats
    cos, sin = M.rotation(positions, D, 10000.0)
    xd = x.double()
    qd, kd, vd = (t.unflatten(1, (-1, D)) for t in (xd @ wqkv.T).split([H * D, K * D, K * D], 1))
    one = torch.ones(1, 0, dtype=torch.float64, device=dev)

    def normed(t, gain, c, s):
        return M.norm_forward(t, gain, c, s, False, 1e-6, torch.float32)[0]

    def dropped(t, i):
        return torch.where(masks[i][0].to(dev).view(T, width), t * masks[i][1], 0.0)
    od = attend(normed(qd, g[0], cos, sin), normed(kd, g[1], cos, sin), vd, cu, cu, D ** -0.5, True)
    h1 = xd + dropped(od.flatten(1) @ wo.T, 0)
    q2 = (h1 @ wq2.T).unflatten(1, (-1, D))
    k2, v2 = (t.unflatten(1, (-1, D)) for t in (e.double() @ wkv.T).split([K * D, K * D], 1))
    none, none_s = one.expand(T, 0), one.expand(S, 0)
    o2 = attend(normed(q2, g[2], none, none), normed(k2, g[3], none_s, none_s), v2, cu, cu_kv, D ** -0.5, False)
    h2 = h1 + dropped(o2.flatten(1) @ wo2.T, 1)
    logp = torch.log_softmax(h2 @ wv.T, 1)
    lp = logp[torch.arange(T, device=dev), y.long()]
    entropy = -(logp.exp() * logp).sum(1)
    # ratios far from the borders, so that no rounding moves a token across one
    delta = torch.tensor([-0.8, -0.05, 0.0, 0.05, 0.8], dtype=torch.float64, device=dev)[torch.randint(0, 5, (T,), generator=gen, device=dev)]
    old, ref = (lp.detach() - delta).float(), (lp.detach() + 0.3 * torch.randn(T, generator=gen, device=dev)).float()
    adv = torch.randn(T, generator=gen, device=dev)
    weight = (torch.arange(T, device=dev) < n).float()
    ratio = (lp - old.double()).exp()
    a = adv.double()
    gap = ref.double() - lp
    each = -torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a) + 0.1 * (gap.exp() - gap - 1) - 0.01 * entropy
    loss = each[:n].sum() / n
    loss.backward()
    want = leaf.grad

    # the program: products by torch, the rest from the library
    wqkv, wo, wq2, wkv, wo2, wv = (m.to(dtype) for m in split(w)[:6])
    g = split(w)[6:]
    rotate, plain = pm.HeadNormRotate(D), pm.HeadNormRotate(D, rotary_dim=0)
    attn, cross, drop, probs = pm.PackedAttention(H, K, D), pm.CrossAttention(H, K, D), pm.Dropout(p), pm.TokenLogProbs(vocab)
    policy = pm.PolicyLoss(clip_low=0.2, clip_high=0.2, kl_coef=0.1, entropy_coef=0.01)
    rngs = [rng, rng + torch.tensor([0, drop.counters(T * width)], device=dev)]
    qkv = x @ wqkv.T
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([H * D, K * D, K * D], 1))
    qn, kn, o = (torch.zeros(T, i, D, dtype=dtype, device=dev) for i in (H, K, H))
    lse, lse2 = torch.zeros(H, T, **f32), torch.zeros(H, T, **f32)
    rotate.pm_head_norm_rotate(q, k, positions, g[0], g[1], qn, kn)
    attn.pm_attention_packed_forward(qn, kn, v, cu, o, lse)
    h1 = torch.zeros_like(x)
    drop.pm_dropout(o.flatten(1) @ wo.T, rngs[0], h1, residual=x)
    q2 = (h1 @ wq2.T).unflatten(1, (-1, D))
    kv = e @ wkv.T
    k2, v2 = (t.unflatten(1, (-1, D)) for t in kv.split([K * D, K * D], 1))
    q2n, k2n, o2 = torch.zeros(T, H, D, dtype=dtype, device=dev), torch.zeros(S, K, D, dtype=dtype, device=dev), torch.zeros(T, H, D, dtype=dtype, device=dev)
    plain.pm_head_norm_rotate(q2, None, None, g[2], None, q2n, None)
    plain.pm_head_norm_rotate(None, k2, None, None, g[3], None, k2n)
    cross.pm_attention_cross_forward(q2n, k2n, v2, cu, cu_kv, o2, lse2)
    h2 = torch.zeros_like(x)
    drop.pm_dropout(o2.flatten(1) @ wo2.T, rngs[1], h2, residual=h1)
    logits = h2 @ wv.T
    got_lp, got_h, row_lse, d_lp, d_h = (torch.zeros(T, **f32) for _ in range(5))
    stats = torch.zeros(5, **f32)
    probs.pm_token_logprobs(logits, y, got_lp, entropy=got_h, lse=row_lse)
    policy.pm_policy_loss(got_lp, old, adv, stats, d_logprob=d_lp, ref_logprob=ref, entropy=got_h, d_entropy=d_h, weight=weight)
    d_logits = torch.zeros_like(logits)
    probs.pm_token_logprobs_backward(logits, y, row_lse, d_logits, d_logprob=d_lp, entropy=got_h, d_entropy=d_h)
    d_h2 = d_logits @ wv
    d_t2, d_t1 = torch.zeros_like(d_h2), torch.zeros_like(d_h2)
    drop.pm_dropout_backward(d_h2, rngs[1], d_t2)
    d_o2 = (d_t2 @ wo2).unflatten(1, (-1, D))
    dq2, dkv = torch.zeros_like(q2n), torch.zeros_like(kv)
    dk2, dv2 = (t.unflatten(1, (-1, D)) for t in dkv.split([K * D, K * D], 1))
    dg = [torch.zeros(D, **f32) for _ in range(4)]
    cross.pm_attention_cross_backward(q2n, k2n, v2, o2, lse2, d_o2, cu, cu_kv, dq2, dk2, dv2)
    plain.pm_head_norm_rotate_backward(q2, None, None, g[2], None, dq2, None, dq2, None, d_q_gain=dg[2])
    plain.pm_head_norm_rotate_backward(None, k2, None, None, g[3], None, dk2, None, dk2, d_k_gain=dg[3])
    d_h1 = d_h2 + dq2.flatten(1) @ wq2
    drop.pm_dropout_backward(d_h1, rngs[0], d_t1)
    d_o = (d_t1 @ wo).unflatten(1, (-1, D))
    d_qkv = torch.zeros_like(qkv)
    dq, dk, dv = (t.unflatten(1, (-1, D)) for t in d_qkv.split([H * D, K * D, K * D], 1))
    attn.pm_attention_packed_backward(qn, kn, v, o, lse, d_o, cu, dq, dk, dv)
    rotate.pm_head_norm_rotate_backward(q, k, positions, g[0], g[1], dq, dk, dq, dk, d_q_gain=dg[0], d_k_gain=dg[1])
    grads = [d_qkv.T @ x, d_t1.T @ o.flatten(1), dq2.flatten(1).T @ h1, dkv.T @ e, d_t2.T @ o2.flatten(1), d_logits.T @ h2, *dg]
    arena, norm, scale = torch.zeros(total, **f32), torch.zeros(1, **f32), torch.zeros(1, **f32)
    pm.GradClip([t.contiguous() for t in grads], [arena[i:i + k] for i, k in zip(starts, sizes)]).pm_clip_gradients(float("inf"), norm, scale)

    # in bf16 every tensor between two products is rounded once, 26 on the longest path, each 2^-8 of its size at most; in fp32 the products'
    # sums of up to 520 terms on as many steps
    tol = 26 * R.u(dtype) if dtype != torch.float32 else 26 * 520 * R.SUM
    assert abs(float(stats[0]) - float(loss.detach())) <= tol * float(each[:n].detach().abs().sum()) / n
    assert float((got_lp[:n].double() - lp.detach()[:n]).abs().max()) <= tol * float(logp.detach().abs().max())
    want_norm = float(want.norm())
    assert abs(float(norm) - want_norm) <= tol * want_norm and float(scale) == 1.0
    for i, (a, k) in enumerate(zip(starts, sizes)):
        part = want[a:a + k]
        assert float((arena[a:a + k].double() - part).norm()) <= 2 * tol * float(part.norm()), i

    # decoding: the last token of each sequence alone gives what it gave among the others
    last = (cu[1:] - 1).long()
    cu1 = torch.arange(4, dtype=torch.int32, device=dev)
    o1, lse1 = torch.zeros(3, H, D, dtype=dtype, device=dev), torch.zeros(H, 3, **f32)
    q1, qn1 = q2[last].contiguous(), torch.zeros(3, H, D, dtype=dtype, device=dev)
    plain.pm_head_norm_rotate(q1, None, None, g[2], None, qn1, None)
    assert torch.equal(qn1, q2n[last])
    cross.pm_attention_cross_forward(qn1, k2n, v2, cu1, cu_kv, o1, lse1)
    wo_, wl, bo, bl = M.cross_forward(qn1, k2n, v2, cu1, cu_kv, D ** -0.5, dtype)
    assert ((o1.double() - wo_).abs() <= bo).all() and ((lse1.double() - wl).abs() <= bl).all()
    assert float((o1.double() - o2[last].double()).abs().max()) <= 2 * float(bo.max()) and float((lse1 - lse2[:, last]).abs().max()) <= 2 * float(bl.max())
    attn.pm_attention_packed_status()
