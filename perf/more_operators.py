"""The operators around `perf/operators.py`'s that an encoder-decoder trained on its own samples needs, as they are timed:
attention of decoder tokens over an encoder's states of another length, norms and rotation of queries and keys, dropout added to
a residual stream, and the clipped policy loss, each with its gradients.

One pass of a cross-attention case is one forward call, one backward call, or both, over a batch of sequences laid end to end;
k and v are views of one projection of the encoder's output, and their gradients are views of one buffer.  A step has a token
or a few (beams) to each sequence.  One pass of a norm case takes the queries and keys of one projection's output to the ones
that attention reads, or their gradients back, or both.  One pass of a dropout case adds what is kept of a layer's output to
the residual stream, or takes the gradient back, or both.  One pass of a policy case computes the loss of a batch of sampled
tokens with the gradients that go back through the log probabilities and the entropies.
Output buffers belong to the program and are kept from call to call.
"""
import math

import numpy as np
import torch

own = False

DROP_BITS = 1 << 16                                          # a kept or dropped element is decided by 16 bits


# ---- the cases -----------------------------------------------------------------------------------------------------

def _cross(what, lens, kv_lens, heads, kv_heads, d_head, compute, tail=0):
    return dict(kind="cross", what=what, lens=",".join(str(n) for n in lens), kv_lens=",".join(str(n) for n in kv_lens), tail=tail,
                heads=heads, kv_heads=kv_heads, d_head=d_head, compute=compute)


def _norm(what, tokens, heads, kv_heads, d_head, compute, rotary=None, interleaved=False, far=0):
    return dict(kind="norm", what=what, tokens=tokens, heads=heads, kv_heads=kv_heads, d_head=d_head, compute=compute,
                rotary=d_head if rotary is None else rotary, interleaved=interleaved, far=far)


def _dropout(what, rows, width, compute, p=0.1, residual=True):
    return dict(kind="dropout", what=what, rows=rows, width=width, compute=compute, p=p, residual=residual)


def _policy(tokens, kl=True, entropy=True, padded=True):
    return dict(kind="policy", tokens=tokens, kl=kl, entropy=entropy, padded=padded)


def listed():
    named = [
        # three short sentences and their translations so far, as a debugging run or a last small batch has them: launches decide
        ("cross_fwd_short", _cross("forward", [5, 1, 12], [17, 3, 46], 8, 8, 64, "bf16")),
        # the decoder of the large encoder-decoder: 16 targets of 256 tokens over sources of 100 to 475, 16 heads of 64
        ("cross_fwd_16x256", _cross("forward", [256] * 16, [100 + 25 * i for i in range(16)], 16, 16, 64, "bf16")),
        # summaries of long documents, four query heads to a key/value head
        ("cross_fwd_long_shared", _cross("forward", [2048, 1025], [8192, 4099], 16, 4, 128, "bf16")),
        # a packed batch of targets and longer sources with padding behind the last, backward
        ("cross_bwd_ragged_shared", _cross("backward", [1500, 700, 33, 257], [4096, 3001, 1025, 500], 16, 4, 128, "bf16", tail=37)),
        # one decoding step of 16 sequences over sources of 251 to 4016 tokens
        ("cross_step", _cross("forward", [1] * 16, [251 * (i + 1) for i in range(16)], 16, 16, 64, "bf16")),
        # fp32 network of the size people debug with: forward and backward, odd lengths, heads of 32, shared heads
        ("cross_train_f32", _cross("both", [50, 65, 1, 77, 96], [96, 30, 128, 1, 77], 4, 2, 32, "f32")),
        # queries and keys of one decoding step of 16 sequences, positions far into a long context
        ("norm_step", _norm("forward", 16, 16, 2, 128, "bf16", far=100_000)),
        # queries and keys of two long packed documents, forward and backward
        ("norm_train_long", _norm("both", 12291, 16, 2, 128, "bf16")),
        # a small fp32 network's layer output
        ("dropout_small", _dropout("both", 96, 200, "f32")),
        # the feed-forward output of a large packed batch into the residual stream and back
        ("dropout_large", _dropout("both", 16384, 1024, "bf16")),
        # the samples of one small rollout
        ("policy_small", _policy(4096)),
        # a large rollout: 256 answers of 4096 tokens
        ("policy_large", _policy(1 << 20)),
    ]
    return [dict(case, name=name) for name, case in named]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_cross(rng):
    step = rng.random() < 0.3
    compute = rng.choice(["bf16", "bf16", "f32"])
    what = "forward" if step else rng.choice(["forward", "backward", "both"])
    longest, kv_longest = (4, 6000) if step else (500, 700) if compute == "f32" else (1500, 3000)
    n = _log_int(rng, 1, 32 if step else 10)
    few = rng.choice([1, 1, 2, 4])
    lens = [few if step else _log_int(rng, 1, longest) for _ in range(n)]
    kv_lens = [_log_int(rng, 1, kv_longest) for _ in range(n)]
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4])
    return _cross(what, lens, kv_lens, heads, kv_heads, rng.choice([32, 64, 64, 80, 128, 128]), compute,
                  tail=rng.choice([0, 0, rng.randrange(1, 100)]))


def draw(rng):
    kind = rng.choice(["cross", "cross", "cross", "norm", "dropout", "policy"])
    if kind == "cross":
        most = max(work(case)["flops"] for case in listed())
        case = _draw_cross(rng)
        while work(case)["flops"] * (8 if case["compute"] == "f32" else 1) > most:
            case = _draw_cross(rng)
        return case
    if kind == "norm":
        kv_heads = rng.choice([1, 2, 4, 8])
        heads, d = kv_heads * rng.choice([1, 2, 4]), rng.choice([32, 64, 64, 80, 128, 128])
        return _norm(rng.choice(["forward", "backward", "both"]), _log_int(rng, 1, min(12000, 30_000_000 // ((heads + kv_heads) * d))), heads, kv_heads, d,
                     rng.choice(["bf16", "bf16", "f32"]), rotary=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3,
                     far=rng.choice([0, 0, 100_000, 1_000_000]))
    if kind == "dropout":
        width = _log_int(rng, 24, 4096)
        return _dropout(rng.choice(["forward", "backward", "both"]), _log_int(rng, 1, max(2, 16_000_000 // width)), width,
                        rng.choice(["bf16", "bf16", "f32"]), p=rng.choice([0.1, 0.1, 0.3, 0.0, 0.015]), residual=rng.random() < 0.75)
    return _policy(_log_int(rng, 10, 1_000_000), kl=rng.random() < 0.7, entropy=rng.random() < 0.5, padded=rng.random() < 0.7)


def _ints(text):
    return [int(n) for n in text.split(",")]


def _size(case):
    return 2 if case["compute"] == "bf16" else 4


def work(case):
    if case["kind"] == "cross":
        size, h, hk, d = _size(case), case["heads"], case["kv_heads"], case["d_head"]
        lens, kv_lens = _ints(case["lens"]), _ints(case["kv_lens"])
        n, m, pairs = sum(lens), sum(kv_lens), sum(a * b for a, b in zip(lens, kv_lens))
        q, kv, stats = n * h * d * size, 2 * m * hk * d * size, 4 * n * h
        forward, backward = 2 * q + kv + stats, 4 * q + 2 * kv + stats
        moved = {"forward": forward, "backward": backward, "both": forward + 2 * q + kv}      # d_o and the three gradients beside the forward pass
        return {"bytes": moved[case["what"]], "flops": {"forward": 4, "backward": 10, "both": 14}[case["what"]] * d * h * pairs}
    if case["kind"] == "norm":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["d_head"]
        steps = {"forward": 2, "backward": 3, "both": 4}[case["what"]]
        return {"bytes": n * steps * _size(case) + 4 * case["tokens"], "flops": {"forward": 8, "backward": 16, "both": 24}[case["what"]] * n}
    if case["kind"] == "dropout":
        n = case["rows"] * case["width"]
        forward = 3 if case["residual"] else 2
        return {"bytes": n * {"forward": forward, "backward": 2, "both": forward + 2}[case["what"]] * _size(case), "flops": 3 * n}
    n = case["tokens"]
    return {"bytes": 4 * n * (4 + (2 if case["entropy"] else 0) + (1 if case["kl"] else 0) + (1 if case["padded"] else 0)), "flops": 20 * n}


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
    dtype = torch.bfloat16 if case.get("compute") == "bf16" else torch.float32
    f32 = dict(dtype=torch.float32, device=dev)
    st = dict(case=case)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if case["kind"] == "cross":
        lens, kv_lens, h, hk, d = _ints(case["lens"]), _ints(case["kv_lens"]), case["heads"], case["kv_heads"], case["d_head"]
        rows, kv_rows = sum(lens) + case["tail"], sum(kv_lens) + case["tail"]
        st["q"], st["kv"] = normal(rows, h, d).to(dtype), normal(kv_rows, 2 * hk * d).to(dtype)
        st["k"], st["v"] = (x.unflatten(1, (hk, d)) for x in st["kv"].split(hk * d, dim=1))
        st["dq"], st["d_kv"] = torch.zeros_like(st["q"]), torch.zeros_like(st["kv"])
        st["dk"], st["dv"] = (x.unflatten(1, (hk, d)) for x in st["d_kv"].split(hk * d, dim=1))
        st["o"], st["lse"] = torch.zeros_like(st["q"]), torch.zeros(h, rows, **f32)
        st["d_o"] = normal(rows, h, d).to(dtype)
        st["cu"] = torch.tensor(_starts(lens), dtype=torch.int32, device=dev)
        st["cu_kv"] = torch.tensor(_starts(kv_lens), dtype=torch.int32, device=dev)
        st["scale"] = d ** -0.5
        if case["what"] == "backward":                       # the forward pass has left its output behind
            o, lse = _plain_cross_forward(st)
            st["o"].copy_(o)
            st["lse"].copy_(lse)
    elif case["kind"] == "norm":
        n, h, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["d_head"]
        qkv = normal(n, (h + 2 * hk) * d).to(dtype)
        st["q"], st["k"] = qkv[:, :h * d].unflatten(1, (h, d)), qkv[:, h * d:(h + hk) * d].unflatten(1, (hk, d))
        if case["far"]:
            st["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device=dev).to(torch.int32)
        else:                                                # two documents end to end
            st["positions"] = torch.cat([torch.arange(n - n // 3, device=dev), torch.arange(n // 3, device=dev)]).to(torch.int32)
        st["q_gain"], st["k_gain"] = 1.0 + 0.1 * normal(d), 1.0 + 0.1 * normal(d)
        st["q_out"], st["k_out"] = torch.zeros(n, h, d, dtype=dtype, device=dev), torch.zeros(n, hk, d, dtype=dtype, device=dev)
        st["d_q_out"], st["d_k_out"] = normal(n, h, d).to(dtype), normal(n, hk, d).to(dtype)
        st["dq"], st["dk"] = torch.zeros_like(st["q_out"]), torch.zeros_like(st["k_out"])
        st["d_q_gain"], st["d_k_gain"] = torch.zeros(d, **f32), torch.zeros(d, **f32)
        st["base"], st["eps"] = 10000.0, 1e-6
    elif case["kind"] == "dropout":
        n, width = case["rows"], case["width"]
        st["x"], st["d_y"] = normal(n, width).to(dtype), normal(n, width).to(dtype)
        st["residual"] = normal(n, width).to(dtype) if case["residual"] else None
        st["y"], st["d_x"] = torch.zeros_like(st["x"]), torch.zeros_like(st["x"])
        # the generator's key and the first counter of this call: a run that is some way on
        st["key"], st["first"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 62), (1 << 33) + 1000003 * (seed % 1000)
        st["rng"] = torch.tensor([st["key"], st["first"]], dtype=torch.int64, device=dev)
    else:
        n = case["tokens"]
        st["old_logprob"] = -torch.rand(n, generator=gen, device=dev) * 4.0
        st["logprob"] = (st["old_logprob"] + 0.2 * normal(n)).clamp(max=0.0)
        st["advantage"] = normal(n)
        st["ref_logprob"] = (st["logprob"] + 0.3 * normal(n)).clamp(max=0.0) if case["kl"] else None
        st["entropy"] = 3.0 * torch.rand(n, generator=gen, device=dev) if case["entropy"] else None
        st["weight"] = (torch.rand(n, generator=gen, device=dev) < 0.9).float() if case["padded"] else None
        st["stats"], st["d_logprob"] = torch.zeros(5, **f32), torch.zeros(n, **f32)
        st["d_entropy"] = torch.zeros(n, **f32) if case["entropy"] else None
        st["clip_low"], st["clip_high"], st["kl_coef"], st["entropy_coef"] = 0.2, 0.28, 0.05, 0.01
    if own:
        import paper_1910_05124_b200 as pm
        if case["kind"] == "cross":
            st["op"] = pm.CrossAttention(case["heads"], case["kv_heads"], case["d_head"], scale=st["scale"])
        elif case["kind"] == "norm":
            st["op"] = pm.HeadNormRotate(case["d_head"], rotary_dim=case["rotary"], base=st["base"], interleaved=case["interleaved"], eps=st["eps"])
        elif case["kind"] == "dropout":
            st["op"] = pm.Dropout(case["p"])
        else:
            st["op"] = pm.PolicyLoss(clip_low=st["clip_low"], clip_high=st["clip_high"], kl_coef=st["kl_coef"] if case["kl"] else 0.0,
                                     entropy_coef=st["entropy_coef"] if case["entropy"] else 0.0)
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _padded(x, cu, longest):
    """[rows, heads, d] packed -> [sequence, heads, position, d] in fp32, zeros behind a sequence's end."""
    cu = cu.long()
    at = torch.arange(longest, device=x.device)
    inside = at < (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return torch.where(inside[:, :, None, None], x[rows].float(), 0.0).transpose(1, 2)


def _packed(x, cu, n, dtype):
    """[sequence, heads, position, d] -> [n rows, heads, d], zeros behind the last sequence."""
    cu = cu.long()
    rows = torch.arange(n, device=x.device)
    seq = torch.searchsorted(cu[1:].contiguous(), rows, right=True).clamp(max=cu.numel() - 2)
    pos = (rows - cu[seq]).clamp(max=x.shape[2] - 1)
    return torch.where((rows < cu[-1])[:, None, None], x.transpose(1, 2)[seq, pos], 0.0).to(dtype)


def _queries(x, st):
    """[rows, heads, d] -> [sequence, kv head, group, position, d]"""
    case = st["case"]
    return _padded(x, st["cu"], max(_ints(case["lens"]))).unflatten(1, (case["kv_heads"], case["heads"] // case["kv_heads"]))


def _scores(st):
    q, longest = _queries(st["q"], st), max(_ints(st["case"]["kv_lens"]))
    k, v = (_padded(st[n], st["cu_kv"], longest).unsqueeze(2) for n in ("k", "v"))
    s = (q @ k.transpose(-1, -2)) * st["scale"]
    keep = torch.arange(longest, device=s.device) < (st["cu_kv"][1:] - st["cu_kv"][:-1])[:, None]
    return q, k, v, s.masked_fill_(~keep[:, None, None, None, :], -math.inf)


def _plain_cross_forward(st):
    q, k, v, s = _scores(st)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o, lse = ((p @ v) / total).flatten(1, 2), (m + total.log()).flatten(1, 2)
    rows = st["q"].shape[0]
    return _packed(o, st["cu"], rows, st["q"].dtype), _packed(lse, st["cu"], rows, torch.float32)[:, :, 0].t().contiguous()


def _plain_cross_backward(st, o, lse):
    q, k, v, s = _scores(st)
    d_o = _queries(st["d_o"], st)
    row = _queries((st["d_o"].float() * o.float()).sum(-1, keepdim=True), st)
    p = s.sub_(_queries(lse.t().unsqueeze(-1), st)).exp_()
    dv = (p.transpose(-1, -2) @ d_o).sum(2)
    ds = (d_o @ v.transpose(-1, -2)).sub_(row).mul_(p).mul_(st["scale"])
    dq, dk = (ds @ k).flatten(1, 2), (ds.transpose(-1, -2) @ q).sum(2)
    rows, kv_rows, dtype = st["q"].shape[0], st["kv"].shape[0], st["q"].dtype
    return _packed(dq, st["cu"], rows, dtype), torch.cat([_packed(g, st["cu_kv"], kv_rows, dtype).flatten(1) for g in (dk, dv)], dim=1)


def _rotation(st):
    """cos and sin [tokens, 1, rotary / 2]; angles of far positions need 64 bits."""
    n = st["case"]["rotary"]
    freq = st["base"] ** (-torch.arange(0, n, 2, device=st["positions"].device, dtype=torch.float64) / n)
    angle = st["positions"].double()[:, None, None] * freq
    return angle.cos().float(), angle.sin().float()


def _rotate(x, cos, sin, case):
    n = case["rotary"]
    if case["interleaved"]:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :n // 2], x[..., n // 2:n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., n:]], dim=-1)


def _plain_norm(st, x, gain):
    x = x.float()
    r = (x.square().mean(-1, keepdim=True) + st["eps"]).rsqrt()
    return _rotate(x * r * gain, *_rotation(st), st["case"])


def _plain_norm_backward(st, x, gain, d_out):
    cos, sin = _rotation(st)
    x, u = x.float(), _rotate(d_out.float(), cos, -sin, st["case"])
    r = (x.square().mean(-1, keepdim=True) + st["eps"]).rsqrt()
    xh, a = x * r, u * gain
    return r * (a - xh * (a * xh).mean(-1, keepdim=True)), (u * xh).double().sum((0, 1)).float()


def _high_low(a, b):
    """The halves of the 64-bit product of two 32-bit numbers, b a constant, held in 64-bit integers."""
    low, high = (a & 0xFFFF) * b, (a >> 16) * b
    mid = (low >> 16) + high
    return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _kept(st):
    """Which elements are kept: 16 bits of Philox4x32-10 each, eight elements to a counter."""
    case = st["case"]
    n = case["rows"] * case["width"]
    at = st["first"] + torch.arange(-(-n // 8), device=st["x"].device)
    c, key = [at & 0xFFFFFFFF, at >> 32, torch.zeros_like(at), torch.zeros_like(at)], [st["key"] & 0xFFFFFFFF, st["key"] >> 32]
    for _ in range(10):
        h0, l0 = _high_low(c[0], 0xD2511F53)
        h1, l1 = _high_low(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    bits = torch.stack([half for word in c for half in (word & 0xFFFF, word >> 16)], dim=1).flatten()[:n]
    dropped = round(case["p"] * DROP_BITS)
    return (bits >= dropped).view(case["rows"], case["width"]), DROP_BITS / (DROP_BITS - dropped)


def _plain_policy(st):
    case, lp = st["case"], st["logprob"]
    delta, a = lp.double() - st["old_logprob"].double(), st["advantage"]          # 64 bits: which side of a border a ratio is on
    w = st["weight"] if case["padded"] else torch.ones_like(lp)
    low, high = delta < math.log1p(-st["clip_low"]), delta > math.log1p(st["clip_high"])
    clipped = (high & (a > 0)) | (low & (a < 0))
    ratio = delta.float().exp()
    bound = torch.where(high, 1.0 + st["clip_high"], 1.0 - st["clip_low"])
    policy = -torch.where(clipped, bound, ratio) * a
    grad = torch.where(clipped, 0.0, -ratio * a)
    total = w.double().sum()
    share = torch.where(total > 0, 1.0 / total, 0.0)

    def mean(x):
        return (w.double() * x.double()).sum() * share

    parts = [mean(policy), torch.zeros_like(share), torch.zeros_like(share), mean(clipped)]
    loss, d_entropy = parts[0], None
    if case["kl"]:
        d = st["ref_logprob"] - lp
        parts[1] = mean(torch.expm1(d.double()) - d.double())
        loss = loss + st["kl_coef"] * parts[1]
        grad = grad - st["kl_coef"] * torch.expm1(d)
    if case["entropy"]:
        parts[2] = mean(st["entropy"])
        loss = loss - st["entropy_coef"] * parts[2]
        d_entropy = -st["entropy_coef"] * w * share.float()
    return dict(stats=torch.stack([loss] + parts).float(), d_logprob=w * share.float() * grad, d_entropy=d_entropy)


def run(st):
    case, what, dtype = st["case"], st["case"].get("what"), st["case"].get("compute")
    out = {}
    if case["kind"] == "cross":
        if own:
            op = st["op"]
            if what != "backward":
                op.pm_attention_cross_forward(st["q"], st["k"], st["v"], st["cu"], st["cu_kv"], st["o"], st["lse"])
            if what != "forward":
                op.pm_attention_cross_backward(st["q"], st["k"], st["v"], st["o"], st["lse"], st["d_o"], st["cu"], st["cu_kv"],
                                               st["dq"], st["dk"], st["dv"])
            o, lse, dq, d_kv = st["o"], st["lse"], st["dq"], st["d_kv"]
        else:
            o, lse = _plain_cross_forward(st) if what != "backward" else (st["o"], st["lse"])
            dq, d_kv = _plain_cross_backward(st, o, lse) if what != "forward" else (None, None)
        if what != "backward":
            out.update(o=o, lse=lse)
        if what != "forward":
            out.update(dq=dq, d_kv=d_kv)
        return out
    if case["kind"] == "norm":
        if own:
            op = st["op"]
            if what != "backward":
                op.pm_head_norm_rotate(st["q"], st["k"], st["positions"], st["q_gain"], st["k_gain"], st["q_out"], st["k_out"])
            if what != "forward":
                op.pm_head_norm_rotate_backward(st["q"], st["k"], st["positions"], st["q_gain"], st["k_gain"], st["d_q_out"], st["d_k_out"],
                                                st["dq"], st["dk"], st["d_q_gain"], st["d_k_gain"])
        names = (("q_out", "k_out") if what != "backward" else ()) + (("dq", "dk", "d_q_gain", "d_k_gain") if what != "forward" else ())
        if own:
            return {n: st[n] for n in names}
        for x in ("q", "k"):
            if what != "backward":
                out[x + "_out"] = _plain_norm(st, st[x], st[x + "_gain"]).to(st[x].dtype)
            if what != "forward":
                d, out[f"d_{x}_gain"] = _plain_norm_backward(st, st[x], st[x + "_gain"], st[f"d_{x}_out"])
                out["d" + x] = d.to(st[x].dtype)
        return {n: out[n] for n in names}
    if case["kind"] == "dropout":
        if own:
            if what != "backward":
                st["op"].pm_dropout(st["x"], st["rng"], st["y"], residual=st["residual"])
                out["y"] = st["y"]
            if what != "forward":
                st["op"].pm_dropout_backward(st["d_y"], st["rng"], st["d_x"])
                out["d_x"] = st["d_x"]
            return out
        kept, scale = _kept(st)
        if what != "backward":
            y = torch.where(kept, st["x"].float() * scale, 0.0)
            out["y"] = (y if st["residual"] is None else y + st["residual"].float()).to(st["x"].dtype)
        if what != "forward":
            out["d_x"] = torch.where(kept, st["d_y"].float() * scale, 0.0).to(st["x"].dtype)
        return out
    if own:
        st["op"].pm_policy_loss(st["logprob"], st["old_logprob"], st["advantage"], st["stats"], d_logprob=st["d_logprob"],
                                ref_logprob=st["ref_logprob"], entropy=st["entropy"], d_entropy=st["d_entropy"], weight=st["weight"])
        return {n: st[n] for n in ("stats", "d_logprob", "d_entropy")}
    return _plain_policy(st)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return dict(cross=_exact_cross, norm=_exact_norm, dropout=_exact_dropout, policy=_exact_policy)[case["kind"]](case, st)


def _exact_cross(case, st):
    q, k, v, d_o = (st[n].double() for n in ("q", "k", "v", "d_o"))
    group, what = case["heads"] // case["kv_heads"], case["what"]
    o, lse = torch.zeros_like(q), torch.zeros(case["heads"], q.shape[0], dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    cu, cu_kv = _starts(_ints(case["lens"])), _starts(_ints(case["kv_lens"]))
    for a, b, x, y in zip(cu, cu[1:], cu_kv, cu_kv[1:]):
        for h in range(case["heads"]):
            g = h // group
            s = torch.einsum("id,jd->ij", q[a:b, h], k[x:y, g]) * st["scale"]
            if what == "backward":                           # of the rounded output and statistics that it is given
                p = torch.exp(s - st["lse"][h, a:b, None].double())
                row = (st["o"][a:b, h].double() * d_o[a:b, h]).sum(1)
            else:
                lse[h, a:b] = torch.logsumexp(s, dim=1)
                p = torch.softmax(s, dim=1)
                o[a:b, h] = p @ v[x:y, g]
                row = (o[a:b, h] * d_o[a:b, h]).sum(1)
            if what != "forward":
                ds = p * (d_o[a:b, h] @ v[x:y, g].T - row[:, None])
                dq[a:b, h] = ds @ k[x:y, g] * st["scale"]
                dk[x:y, g] += ds.T @ q[a:b, h] * st["scale"]
                dv[x:y, g] += p.T @ d_o[a:b, h]
            del s, p
    out = dict(o=o, lse=lse) if what != "backward" else {}
    if what != "forward":
        out.update(dq=dq, d_kv=torch.cat([dk.flatten(1), dv.flatten(1)], dim=1))
    return out


def _exact_norm(case, st):
    half, d = case["rotary"] // 2, case["d_head"]
    dev = st["q"].device
    pair = torch.arange(half, device=dev)
    first = 2 * pair if case["interleaved"] else pair
    second = first + 1 if case["interleaved"] else pair + half
    turn = torch.polar(torch.ones(case["tokens"], 1, half, dtype=torch.float64, device=dev),
                       st["positions"].double()[:, None, None] * torch.exp(-(math.log(st["base"]) / half) * pair.double()))
    out = {}
    for x in ("q", "k"):
        leaf, gain = st[x].double().requires_grad_(), st[x + "_gain"].double().requires_grad_()
        normed = leaf / torch.sqrt(leaf.pow(2).sum(-1, keepdim=True) / d + st["eps"]) * gain
        z = torch.complex(normed[..., first], normed[..., second]) * turn
        y = normed.index_copy(-1, first, z.real).index_copy(-1, second, z.imag)
        out[x + "_out"] = y.detach()
        if case["what"] != "forward":
            out["d" + x], out[f"d_{x}_gain"] = torch.autograd.grad(y, (leaf, gain), st[f"d_{x}_out"].double())
    names = (("q_out", "k_out") if case["what"] != "backward" else ()) + (("dq", "dk", "d_q_gain", "d_k_gain") if case["what"] != "forward" else ())
    return {n: out[n] for n in names}


def _exact_dropout(case, st):
    """Philox4x32-10 in numpy's wrapping 64-bit products."""
    n = case["rows"] * case["width"]
    low32, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    at = np.uint64(st["first"]) + np.arange(-(-n // 8), dtype=np.uint64)
    x, y, z, w = at & low32, at >> shift, np.zeros_like(at), np.zeros_like(at)
    ka, kb = st["key"] & 0xFFFFFFFF, st["key"] >> 32
    for i in range(10):
        a, b = x * np.uint64(0xD2511F53), z * np.uint64(0xCD9E8D57)
        x, y, z, w = ((b >> shift) ^ y ^ np.uint64((ka + i * 0x9E3779B9) & 0xFFFFFFFF), b & low32,
                      (a >> shift) ^ w ^ np.uint64((kb + i * 0xBB67AE85) & 0xFFFFFFFF), a & low32)
    words = np.stack([x, y, z, w], axis=1).astype("<u4")
    bits = np.ascontiguousarray(words).view("<u2").reshape(-1)[:n]             # the lower half of a word first
    dropped = int(math.floor(case["p"] * DROP_BITS + 0.5))
    factor = torch.from_numpy((bits >= dropped).astype(np.float64)).to(st["x"].device).view(case["rows"], case["width"]) / (1.0 - dropped / DROP_BITS)
    out = {}
    if case["what"] != "backward":
        out["y"] = factor * st["x"].double() + (0.0 if st["residual"] is None else st["residual"].double())
    if case["what"] != "forward":
        out["d_x"] = factor * st["d_y"].double()
    return out


def _exact_policy(case, st):
    lp = st["logprob"].double().requires_grad_()
    w = st["weight"].double() if case["padded"] else torch.ones_like(lp)
    share = w / w.sum() if float(w.sum()) > 0 else w
    a, ratio = st["advantage"].double(), torch.exp(lp - st["old_logprob"].double())
    free, held = ratio * a, torch.minimum(torch.maximum(ratio, torch.full_like(ratio, 1 - st["clip_low"])),
                                          torch.full_like(ratio, 1 + st["clip_high"])) * a
    zero = torch.zeros((), dtype=torch.float64, device=lp.device)
    parts = [(share * -torch.where(free <= held, free, held)).sum(), zero, zero, (share * (held < free)).sum()]
    loss = parts[0]
    if case["kl"]:
        gap = st["ref_logprob"].double() - lp
        parts[1] = (share * (torch.exp(gap) - gap - 1)).sum()
        loss = loss + st["kl_coef"] * parts[1]
    if case["entropy"]:
        parts[2] = (share * st["entropy"].double()).sum()
        loss = loss - st["entropy_coef"] * parts[2]
    grad, = torch.autograd.grad(loss, lp)
    return dict(stats=torch.stack([loss.detach()] + [p.detach() for p in parts]), d_logprob=grad,
                d_entropy=-st["entropy_coef"] * share if case["entropy"] else None)
