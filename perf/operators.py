"""The operators that a program with its own forward and backward pass calls next to `pm_update_flat`, as they are timed:
attention over packed sequences, log probabilities of given tokens, and gradient clipping, each with its gradients.

One pass of an attention case is one forward call, one backward call, or both, over a batch of sequences laid end to end;
q, k and v are views of one projection's output, and their gradients are views of one buffer.  One pass of a log-probability
case is a forward call (a sampling step, an evaluation), a backward call, or both.  One pass of a clipping case takes the
gradient tensors of a network through the norm and into the slices of the fp32 gradient arena that the update reads.
Output buffers belong to the program and are kept from call to call.
"""
import math

import torch

own = False


# ---- the cases -----------------------------------------------------------------------------------------------------

def _attention(what, lens, heads, kv_heads, d_head, compute, tail=0, causal=True):
    return dict(kind="attention", what=what, lens=",".join(str(n) for n in lens), tail=tail, heads=heads, kv_heads=kv_heads,
                d_head=d_head, compute=compute, causal=causal)


def _logprob(what, rows, vocab, compute, top_k=0, entropy=True, padded=False):
    return dict(kind="logprob", what=what, rows=rows, vocab=vocab, compute=compute, top_k=top_k, entropy=entropy, padded=padded)


def _clip(layers, width, d_ff, vocab, compute, clips=True):
    return dict(kind="clip", layers=layers, width=width, d_ff=d_ff, vocab=vocab, compute=compute, clips=clips)


def listed():
    named = [
        # three short sentences, one of a single token, as a debugging run or a last small batch has them: launches decide
        ("attn_fwd_short", _attention("forward", [17, 1, 46], 8, 8, 64, "bf16")),
        # the decoder of the large encoder-decoder: 16 sequences of 256 tokens, 16 heads of 64
        ("attn_fwd_16x256", _attention("forward", [256] * 16, 16, 16, 64, "bf16")),
        # long documents, four query heads to a key/value head
        ("attn_fwd_long_shared", _attention("forward", [8192, 4099], 16, 4, 128, "bf16")),
        # the backward pass of the decoder
        ("attn_bwd_16x256", _attention("backward", [256] * 16, 16, 16, 64, "bf16")),
        # a packed batch of long and short documents with padding behind the last, backward
        ("attn_bwd_ragged_shared", _attention("backward", [4096, 3001, 1025, 500, 33], 16, 4, 128, "bf16", tail=37)),
        # fp32 network of the size people debug with: forward and backward, odd lengths, heads of 32, shared heads
        ("attn_train_f32", _attention("both", [96, 65, 128, 1, 77, 30, 96], 4, 2, 32, "f32")),
        # one sampling step of 16 sequences: log probability, entropy and the eight best of 32000 logits each
        ("logprob_step", _logprob("forward", 16, 32000, "f32", top_k=8)),
        # an evaluation pass over the large encoder-decoder's microbatch
        ("logprob_eval", _logprob("forward", 4096, 32000, "f32", top_k=8)),
        # the gradient of that microbatch's loss and entropy bonus, bf16 logits
        ("logprob_bwd_bf16", _logprob("backward", 4096, 32000, "bf16")),
        # loss and gradient over a vocabulary that no vector length divides, with padded targets
        ("logprob_train_ragged", _logprob("both", 1345, 8191, "f32", entropy=False, padded=True)),
        # gradients of the smallest network that is trained in earnest
        ("clip_small", _clip(2, 128, 512, 1000, "f32")),
        # gradients of an encoder-decoder of the large widths at 4 + 4 layers, bf16 into the fp32 arena
        ("clip_large", _clip(12, 1024, 4096, 32000, "bf16")),
    ]
    return [dict(case, name=name) for name, case in named]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "logprob", "clip"])
    if kind == "attention":
        compute = rng.choice(["bf16", "bf16", "f32"])
        what = rng.choice(["forward", "backward", "both"])
        longest = _log_int(rng, 4, 700 if compute == "f32" else 4096 if what == "forward" else 2048)
        lens, room = [], 5000 if compute == "bf16" else 1400
        for _ in range(_log_int(rng, 1, 12)):
            n = min(_log_int(rng, 1, longest), room)
            if n > 0:
                lens.append(n)
                room -= n
        kv_heads = rng.choice([1, 2, 4])
        heads = kv_heads * rng.choice([1, 2, 4])
        return _attention(what, lens, heads, kv_heads, rng.choice([32, 64, 64, 80, 128, 128]),
                          compute, tail=rng.choice([0, 0, rng.randrange(1, 100)]), causal=rng.random() < 0.75)
    if kind == "logprob":
        vocab = _log_int(rng, 50, 60000)
        rows = _log_int(rng, 1, max(2, min(6000, 60_000_000 // vocab)))
        return _logprob(rng.choice(["forward", "backward", "both"]), rows, vocab, rng.choice(["f32", "bf16"]),
                        top_k=rng.choice([0, 1, 5, 8, 20]), entropy=rng.random() < 0.5, padded=rng.random() < 0.5)
    width = _log_int(rng, 24, 1000)
    return _clip(_log_int(rng, 1, 12), width, 4 * width + rng.choice([0, 1, 8]), _log_int(rng, 50, 32000),
                 rng.choice(["f32", "bf16", "mixed"]), clips=rng.random() < 0.75)


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _pairs(case):
    return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lens(case))


def _clip_sizes(case):
    """Element counts of the gradient tensors: the embedding, per layer the projections, the feed-forward pair, two layer norms."""
    d, f = case["width"], case["d_ff"]
    sizes = [case["vocab"] * d]
    for _ in range(case["layers"]):
        sizes += [d * d, d] * 4 + [d * f, f, f * d, d, d, d, d, d]
    return sizes


def _clip_dtypes(case, sizes):
    if case["compute"] == "mixed":                           # matrices in bf16, biases and layer norms in fp32
        return [torch.bfloat16 if n >= case["width"] ** 2 else torch.float32 for n in sizes]
    return [torch.bfloat16 if case["compute"] == "bf16" else torch.float32] * len(sizes)


def work(case):
    if case["kind"] == "attention":
        size = 2 if case["compute"] == "bf16" else 4
        n, h, hk, d = sum(_lens(case)), case["heads"], case["kv_heads"], case["d_head"]
        moved = {"forward": (2 * h + 2 * hk) * d * size + 4 * h, "backward": (4 * h + 4 * hk) * d * size + 4 * h}
        moved["both"] = moved["forward"] + moved["backward"] - (2 * h + 2 * hk) * d * size - 4 * h
        per = {"forward": 4, "backward": 10, "both": 14}
        return {"bytes": n * moved[case["what"]], "flops": per[case["what"]] * d * _pairs(case) * h}
    if case["kind"] == "logprob":
        size = 2 if case["compute"] == "bf16" else 4
        n, v = case["rows"], case["vocab"]
        moved = {"forward": n * v * size, "backward": 2 * n * v * size, "both": 2 * n * v * size}[case["what"]]
        return {"bytes": moved + n * (16 + 8 * case["top_k"]), "flops": {"forward": 5, "backward": 5, "both": 10}[case["what"]] * n * v}
    sizes = _clip_sizes(case)
    dtypes = _clip_dtypes(case, sizes)
    return {"bytes": sum(n * (t.itemsize + 4) for n, t in zip(sizes, dtypes)), "flops": 3 * sum(sizes)}


# ---- what a program has in hand -------------------------------------------------------------------------------------

def _starts(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(dev)
    gen.manual_seed(seed)
    dtype = torch.bfloat16 if case["compute"] == "bf16" else torch.float32
    st = dict(case=case)
    if case["kind"] == "attention":
        lens, h, hk, d = _lens(case), case["heads"], case["kv_heads"], case["d_head"]
        rows = sum(lens) + case["tail"]
        qkv = torch.randn(rows, (h + 2 * hk) * d, generator=gen, device=dev).to(dtype)
        d_qkv = torch.zeros(rows, (h + 2 * hk) * d, dtype=dtype, device=dev)
        st["q"], st["k"], st["v"] = _heads(qkv, case)
        st["dq"], st["dk"], st["dv"] = _heads(d_qkv, case)
        st["d_qkv"] = d_qkv
        st["o"] = torch.zeros(rows, h, d, dtype=dtype, device=dev)
        st["lse"] = torch.zeros(h, rows, device=dev)
        st["d_o"] = torch.randn(rows, h, d, generator=gen, device=dev).to(dtype)
        st["cu_seqlens"] = torch.tensor(_starts(lens), dtype=torch.int32, device=dev)
        st["longest"] = max(lens)
        st["scale"] = d ** -0.5
        if case["what"] == "backward":                       # the forward pass has left its output behind
            o, lse = _plain_attention_forward(st)
            st["o"].copy_(o)
            st["lse"].copy_(lse)
    elif case["kind"] == "logprob":
        n, v = case["rows"], case["vocab"]
        st["logits"] = (3.0 * torch.randn(n, v, generator=gen, device=dev)).to(dtype)
        st["targets"] = torch.randint(0, v, (n,), generator=gen, device=dev).to(torch.int32)
        if case["padded"]:
            st["targets"][torch.rand(n, generator=gen, device=dev) < 0.05] = -1
        f32 = dict(dtype=torch.float32, device=dev)
        st["logprob"], st["lse"] = torch.zeros(n, **f32), torch.zeros(n, **f32)
        st["entropy"] = torch.zeros(n, **f32) if case["entropy"] else None
        k = case["top_k"]
        st["top_logprob"] = torch.zeros(n, k, **f32) if k else None
        st["top_ids"] = torch.zeros(n, k, dtype=torch.int32, device=dev) if k else None
        if case["what"] != "forward":
            st["d_logprob"] = torch.randn(n, generator=gen, device=dev) / n
            st["d_entropy"] = torch.randn(n, generator=gen, device=dev) / n if case["entropy"] else None
            st["d_logits"] = torch.zeros(n, v, dtype=dtype, device=dev)
        if case["what"] == "backward":
            logprob, entropy, lse, _, _ = _plain_logprobs(st)
            st["lse"].copy_(lse)
            if case["entropy"]:
                st["entropy"].copy_(entropy)
    else:
        sizes = _clip_sizes(case)
        scale = 1.0 / math.sqrt(sum(sizes))                  # a norm of about one
        st["grads"] = [(scale * torch.randn(n, generator=gen, device=dev)).to(t) for n, t in zip(sizes, _clip_dtypes(case, sizes))]
        padded = [-(-n // 64) * 64 for n in sizes]           # slices of the arena start at multiples of 64 elements
        st["padded"] = padded
        st["arena"] = torch.zeros(sum(padded), device=dev)
        st["outs"] = [st["arena"][a:a + n] for a, n in zip(_starts(padded), sizes)]
        st["max_norm"] = 0.25 if case["clips"] else 25.0
        st["norm"], st["scale"] = torch.zeros(1, device=dev), torch.zeros(1, device=dev)
    if own:
        import paper_1910_05124_b200 as pm
        if case["kind"] == "attention":
            st["op"] = pm.PackedAttention(case["heads"], case["kv_heads"], case["d_head"], causal=case["causal"], scale=st["scale"])
        elif case["kind"] == "logprob":
            st["op"] = pm.TokenLogProbs(case["vocab"], top_k=case["top_k"])
        else:
            st["op"] = pm.GradClip(st["grads"], st["outs"])
    return st


def _heads(buffer, case):
    h, hk, d = case["heads"], case["kv_heads"], case["d_head"]
    q, k, v = buffer.split([h * d, hk * d, hk * d], dim=1)
    return q.unflatten(1, (h, d)), k.unflatten(1, (hk, d)), v.unflatten(1, (hk, d))


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _padded(x, st):
    """[rows, heads, d] packed -> [sequence, heads, position, d] in fp32, zeros behind a sequence's end."""
    cu = st["cu_seqlens"].long()
    at = torch.arange(st["longest"], device=x.device)
    inside = at < (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return torch.where(inside[:, :, None, None], x[rows].float(), 0.0).transpose(1, 2)


def _packed(x, st, dtype):
    """[sequence, heads, position, d] -> [rows, heads, d], zeros behind the last sequence."""
    cu = st["cu_seqlens"].long()
    rows = torch.arange(st["q"].shape[0], device=x.device)
    seq = torch.searchsorted(cu[1:].contiguous(), rows, right=True).clamp(max=cu.numel() - 2)
    pos = (rows - cu[seq]).clamp(max=st["longest"] - 1)
    return torch.where((rows < cu[-1])[:, None, None], x.transpose(1, 2)[seq, pos], 0.0).to(dtype)


def _scores(st):
    """q, k, v as [sequence, kv head, group, position, d] and the masked scores."""
    case = st["case"]
    group = case["heads"] // case["kv_heads"]
    q = _padded(st["q"], st).unflatten(1, (case["kv_heads"], group))
    k, v = _padded(st["k"], st).unsqueeze(2), _padded(st["v"], st).unsqueeze(2)
    s = (q @ k.transpose(-1, -2)) * st["scale"]
    cu = st["cu_seqlens"]
    at = torch.arange(st["longest"], device=s.device)
    keep = (at < (cu[1:] - cu[:-1])[:, None])[:, None, None, None, :]
    if case["causal"]:
        keep = keep & (at[None, :] <= at[:, None])
    return q, k, v, s.masked_fill_(~keep, -math.inf)


def _plain_attention_forward(st):
    q, k, v, s = _scores(st)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / total
    lse = (m + total.log()).flatten(1, 2)
    return _packed(o.flatten(1, 2), st, st["q"].dtype), _packed(lse, st, torch.float32)[:, :, 0].t().contiguous()


def _plain_attention_backward(st, o, lse):
    case = st["case"]
    group = case["heads"] // case["kv_heads"]
    q, k, v, s = _scores(st)
    d_o = _padded(st["d_o"], st).unflatten(1, (case["kv_heads"], group))
    row = (st["d_o"].float() * o.float()).sum(-1, keepdim=True)
    row = _padded(row, st).unflatten(1, (case["kv_heads"], group))
    lse = _padded(lse.t().unsqueeze(-1), st).unflatten(1, (case["kv_heads"], group))
    p = s.sub_(lse).exp_()
    dv = (p.transpose(-1, -2) @ d_o).sum(2)
    ds = (d_o @ v.transpose(-1, -2)).sub_(row).mul_(p).mul_(st["scale"])
    dq = (ds @ k).flatten(1, 2)
    dk = (ds.transpose(-1, -2) @ q).sum(2)
    return torch.cat([_packed(g, st, st["q"].dtype).flatten(1) for g in (dq, dk, dv)], dim=1)


def _plain_logprobs(st):
    x, k = st["logits"].float(), st["case"]["top_k"]
    m = x.amax(1)
    e = (x - m[:, None]).exp()
    total = e.sum(1)
    lse = m + total.log()
    y = st["targets"].long()
    logprob = (x.gather(1, y.clamp(min=0)[:, None])[:, 0] - m) - total.log()
    logprob = torch.where(y < 0, 0.0, logprob)
    entropy = total.log() - (e * (x - m[:, None])).sum(1) / total if st["case"]["entropy"] else None
    if not k:
        return logprob, entropy, lse, None, None
    # one whole number that orders by value and, among equal values, by the lower place
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) - torch.arange(x.shape[1], device=x.device)
    ids = key.topk(k, dim=1).indices
    return logprob, entropy, lse, (x.gather(1, ids) - m[:, None]) - total.log()[:, None], ids.to(torch.int32)


def _plain_logprobs_backward(st, entropy, lse):
    x, y, g = st["logits"].float(), st["targets"].long(), st["d_logprob"]
    g = torch.where(y < 0, 0.0, g)
    logp = x - lse[:, None]
    p = logp.exp()
    dx = -g[:, None] * p
    if st["case"]["entropy"]:
        dx -= st["d_entropy"][:, None] * p * (logp + entropy[:, None])
    dx.scatter_add_(1, y.clamp(min=0)[:, None], g[:, None])
    return dx.to(st["logits"].dtype)


def _plain_clip(st):
    flat = torch.cat([x for g, n in zip(st["grads"], st["padded"]) for x in (g.float(), g.new_zeros(n - g.numel(), dtype=torch.float32))])
    norm = flat.double().square().sum().sqrt()
    scale = torch.clamp(st["max_norm"] / norm, max=1.0)
    return norm.float().reshape(1), scale.float().reshape(1), flat * scale.float()


def run(st):
    case = st["case"]
    if case["kind"] == "attention":
        if own:
            op = st["op"]
            if case["what"] != "backward":
                op.pm_attention_packed_forward(st["q"], st["k"], st["v"], st["cu_seqlens"], st["o"], st["lse"])
            if case["what"] != "forward":
                op.pm_attention_packed_backward(st["q"], st["k"], st["v"], st["o"], st["lse"], st["d_o"], st["cu_seqlens"],
                                                st["dq"], st["dk"], st["dv"])
            o, lse, d_qkv = st["o"], st["lse"], st["d_qkv"]
        else:
            o, lse = _plain_attention_forward(st) if case["what"] != "backward" else (st["o"], st["lse"])
            d_qkv = _plain_attention_backward(st, o, lse) if case["what"] != "forward" else None
        return {"forward": dict(o=o, lse=lse), "backward": dict(d_qkv=d_qkv), "both": dict(o=o, lse=lse, d_qkv=d_qkv)}[case["what"]]
    if case["kind"] == "logprob":
        if own:
            op = st["op"]
            if case["what"] != "backward":
                op.pm_token_logprobs(st["logits"], st["targets"], st["logprob"], entropy=st["entropy"], lse=st["lse"],
                                     top_logprob=st["top_logprob"], top_ids=st["top_ids"])
            if case["what"] != "forward":
                op.pm_token_logprobs_backward(st["logits"], st["targets"], st["lse"], st["d_logits"], d_logprob=st["d_logprob"],
                                              entropy=st["entropy"], d_entropy=st["d_entropy"])
            out, d_logits = [st[n] for n in ("logprob", "entropy", "lse", "top_logprob", "top_ids")], st.get("d_logits")
        else:
            out = _plain_logprobs(st) if case["what"] != "backward" else (None, st["entropy"], st["lse"], None, None)
            d_logits = _plain_logprobs_backward(st, out[1], out[2]) if case["what"] != "forward" else None
        if case["what"] == "backward":
            return dict(d_logits=d_logits)
        return dict(zip(("logprob", "entropy", "lse", "top_logprob", "top_ids"), out), d_logits=d_logits)
    if own:
        st["op"].pm_clip_gradients(st["max_norm"], st["norm"], st["scale"])
        return dict(norm=st["norm"], scale=st["scale"], arena=st["arena"])
    return dict(zip(("norm", "scale", "arena"), _plain_clip(st)))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, st)
    if case["kind"] == "logprob":
        return _exact_logprob(case, st)
    total = sum(float(g.double().pow(2).sum()) for g in st["grads"])
    norm = math.sqrt(total)
    scale = min(1.0, st["max_norm"] / norm)
    arena = torch.zeros(sum(st["padded"]), dtype=torch.float64, device=st["arena"].device)
    at = 0
    for g, n in zip(st["grads"], st["padded"]):
        arena[at:at + g.numel()] = g.double() * scale
        at += n
    one = dict(dtype=torch.float64)
    return dict(norm=torch.tensor([norm], **one), scale=torch.tensor([scale], **one), arena=arena)


def _exact_attention(case, st):
    q, k, v, d_o = (st[n].double() for n in ("q", "k", "v", "d_o"))
    group, what = case["heads"] // case["kv_heads"], case["what"]
    o = torch.zeros_like(q)
    lse = torch.zeros(case["heads"], q.shape[0], dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    cu = _starts(_lens(case))
    for a, b in zip(cu, cu[1:]):
        for h in range(case["heads"]):
            g = h // group
            s = torch.einsum("id,jd->ij", q[a:b, h], k[a:b, g]) * st["scale"]
            if case["causal"]:
                s = s + torch.full_like(s, -math.inf).triu(1)
            if what == "backward":                           # of the rounded output and statistics that it is given
                p = torch.exp(s - st["lse"][h, a:b, None].double())
                row = (st["o"][a:b, h].double() * d_o[a:b, h]).sum(1)
            else:
                lse[h, a:b] = torch.logsumexp(s, dim=1)
                p = torch.softmax(s, dim=1)
                o[a:b, h] = p @ v[a:b, g]
                row = (o[a:b, h] * d_o[a:b, h]).sum(1)
            if what != "forward":
                ds = p * (d_o[a:b, h] @ v[a:b, g].T - row[:, None])
                dq[a:b, h] = ds @ k[a:b, g] * st["scale"]
                dk[a:b, g] += ds.T @ q[a:b, h] * st["scale"]
                dv[a:b, g] += p.T @ d_o[a:b, h]
            del s, p
    d_qkv = torch.cat([g.flatten(1) for g in (dq, dk, dv)], dim=1)
    return {"forward": dict(o=o, lse=lse), "backward": dict(d_qkv=d_qkv), "both": dict(o=o, lse=lse, d_qkv=d_qkv)}[what]


def _exact_logprob(case, st):
    n, k, what = case["rows"], case["top_k"], case["what"]
    y = st["targets"].long()
    out = {name: [] for name in ("logprob", "entropy", "lse", "top_logprob", "top_ids", "d_logits")}
    for a in range(0, n, 512):                               # some rows at a time
        rows = slice(a, min(n, a + 512))
        x, t = st["logits"][rows].double(), y[rows]
        logp = torch.log_softmax(x, dim=1)
        if what == "backward":
            logp = x - st["lse"][rows, None].double()
        p = logp.exp()
        entropy = -(p * logp).sum(1)
        if what == "backward" and case["entropy"]:
            entropy = st["entropy"][rows].double()
        place = torch.arange(x.shape[0], device=x.device)
        out["logprob"].append(torch.where(t < 0, 0.0, logp[place, t.clamp(min=0)]))
        out["entropy"].append(entropy)
        out["lse"].append(torch.logsumexp(x, dim=1))
        if k:
            best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
            out["top_ids"].append(best.to(torch.int32))
            out["top_logprob"].append(logp.gather(1, best))
        if what != "forward":
            g = torch.where(t < 0, 0.0, st["d_logprob"][rows].double())
            dx = -g[:, None] * p
            if case["entropy"]:
                dx = dx - st["d_entropy"][rows, None].double() * p * (logp + entropy[:, None])
            dx[place, t.clamp(min=0)] += g
            out["d_logits"].append(dx)
    got = {name: torch.cat(parts) if parts else None for name, parts in out.items()}
    if not case["entropy"]:
        got["entropy"] = None
    return dict(d_logits=got["d_logits"]) if what == "backward" else got
