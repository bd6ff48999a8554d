"""The operators as a program uses them: one training step of a small causal language model over packed sequences, from its
embedded tokens to the fused update, against the same step in 64 bits."""
import pytest
import torch

import operators_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_step(cuda_device, dtype):
    import paper_1910_05124_b200 as pm
    dev = cuda_device
    gen = torch.Generator(dev).manual_seed(1)
    H, K, D, vocab, lens, tail = 4, 2, 64, 518, [37, 1, 90], 6
    width, T = 96, sum(lens) + tail
    cu = R.lens_to_cu(lens, dev)
    shapes = [((H + 2 * K) * D, width), (width, H * D), (vocab, width)]           # projection, output, vocabulary
    sizes = [a * b for a, b in shapes]
    starts = [0, sizes[0], sizes[0] + sizes[1]]
    total = sum(sizes)
    assert all(n % 64 == 0 for n in sizes)
    w = torch.randn(total, generator=gen, device=dev) * 0.1
    x = torch.randn(T, width, generator=gen, device=dev).to(dtype)
    y = torch.randint(0, vocab, (T,), generator=gen, device=dev).to(torch.int32)
    y[sum(lens):] = -1
    n_real = sum(lens)

    def split(flat):
        return [flat[a:a + n].view(s) for a, n, s in zip(starts, sizes, shapes)]
    # the program: products by torch, the rest from the library
    wq, wo, wv = (m.to(dtype) for m in split(w))
    attn, loss, f32 = pm.PackedAttention(H, K, D), pm.TokenLogProbs(vocab, top_k=3), dict(dtype=torch.float32, device=dev)
    qkv = x @ wq.T
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([H * D, K * D, K * D], 1))
    o, lse = torch.zeros(T, H, D, dtype=dtype, device=dev), torch.zeros(H, T, **f32)
    attn.pm_attention_packed_forward(q, k, v, cu, o, lse)
    h = x + o.flatten(1) @ wo.T
    logits = h @ wv.T
    logprob, entropy, row_lse = (torch.zeros(T, **f32) for _ in range(3))
    top, ids = torch.zeros(T, 3, **f32), torch.zeros(T, 3, dtype=torch.int32, device=dev)
    loss.pm_token_logprobs(logits, y, logprob, entropy=entropy, lse=row_lse, top_logprob=top, top_ids=ids)
    gl = torch.full((T,), -1.0 / n_real, **f32)
    gh = torch.where(y < 0, 0.0, -0.01 / n_real).to(torch.float32)                 # an entropy bonus
    d_logits = torch.zeros_like(logits)
    loss.pm_token_logprobs_backward(logits, y, row_lse, d_logits, d_logprob=gl, entropy=entropy, d_entropy=gh)
    d_h = d_logits @ wv
    d_o = (d_h @ wo).unflatten(1, (-1, D))
    d_qkv = torch.zeros_like(qkv)
    dq, dk, dv = (t.unflatten(1, (-1, D)) for t in d_qkv.split([H * D, K * D, K * D], 1))
    attn.pm_attention_packed_backward(q, k, v, o, lse, d_o, cu, dq, dk, dv)
    grads = [d_qkv.T @ x, d_h.T @ o.flatten(1), d_logits.T @ h]
    arena, norm, scale = torch.zeros(total, **f32), torch.zeros(1, **f32), torch.zeros(1, **f32)
    pm.GradClip([g.contiguous() for g in grads], [arena[a:a + n] for a, n in zip(starts, sizes)]).pm_clip_gradients(0.05, norm, scale)
    before = w.clone()
    m, delta = torch.zeros(total, **f32), torch.zeros(total, **f32)
    up = pm.FlatUpdate(starts, sizes, [1, 1, 1], [0, 0, 0], optimizer="sgdm", alpha=0.1, t1=False, t2=False)
    up.pm_update_flat(w, m, None, delta, arena, None, 0)

    # the same step in 64 bits by automatic differentiation
    leaf = before.double().requires_grad_()
    pq, po, pv = split(leaf)
    if dtype != torch.float32:                                # of the rounded weights
        pq, po, pv = (a + (b.double() - a).detach() for a, b in zip((pq, po, pv), (wq, wo, wv)))
    xd = x.double()
    qd, kd, vd = (t.unflatten(1, (-1, D)) for t in (xd @ pq.T).split([H * D, K * D, K * D], 1))
    rows = []
    for a, b in R.spans(cu):
        heads = []
        for i in range(H):
            s = (qd[a:b, i] @ kd[a:b, i // 2].T) * D ** -0.5
            s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
            heads.append(torch.softmax(s, 1) @ vd[a:b, i // 2])
        rows.append(torch.stack(heads, 1))
    od = torch.cat(rows + [torch.zeros(tail, H, D, dtype=torch.float64, device=dev)])
    ld = torch.log_softmax((xd + od.flatten(1) @ po.T) @ pv.T, 1)
    want_lp = ld[torch.arange(T, device=dev), y.long().clamp(min=0)]
    want_h = -(ld.exp() * ld).sum(1)
    (-(want_lp[:n_real]).sum() / n_real - 0.01 * want_h[:n_real].sum() / n_real).backward()
    want = leaf.grad
    want_norm = float(want.norm())
    # in bf16 every tensor between two products is rounded once, about ten on the longest path, each 2^-8 of its size at most; in
    # fp32 the products' sums of up to 518 terms
    tol = 10 * R.u(dtype) if dtype != torch.float32 else 518 * R.SUM
    assert abs(float(norm) - want_norm) <= tol * want_norm
    clipped = want * (0.05 / want_norm)
    assert want_norm > 0.05 and float((arena.double() - clipped).norm()) <= 2 * tol * 0.05
    assert float((w - before + 0.1 * arena).abs().max()) <= 2 * R.U32 * float(before.abs().max())
    far = (logprob[:n_real].double() - want_lp[:n_real]).abs().max()
    assert float(far.detach()) <= tol * float(ld.detach().abs().max()) and (logprob[n_real:] == 0).all()
    assert float((entropy[:n_real].double() - want_h.detach()[:n_real]).abs().max()) <= tol * float(want_h.detach().max()) * 2
    assert torch.equal(ids, R.logprobs(logits, None, 3)["top_ids"])
