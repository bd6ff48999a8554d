"""Plain 64-bit forms of the stand-alone operators, with bounds on how far a correct fp32 or bf16 implementation may be off.

u(t) is the largest relative error of one rounding to type t.  Sums in fp32 are given 2 u(fp32) per addition, which also covers
an accumulator that truncates."""
import math

import torch

U32 = 2.0 ** -24
SUM = 2 * U32
TINY = 2.0 ** -126


def u(dtype):
    return torch.finfo(dtype).eps / 2


def lens_to_cu(lens, device, first=0):
    cu = [first]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=device)


def spans(cu):
    c = cu.tolist()
    return list(zip(c, c[1:]))


def _scores(q, k, scale, causal):
    s = (q @ k.T) * scale
    if causal:
        s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -math.inf)
    return s


def _score_error(q, k, scale):
    """Largest absolute error of a score: d products summed, one product with the scale, the subtraction of a maximum or lse, and
    the exponential's argument times log2(e), of arguments up to the largest score."""
    d = q.shape[1]
    most = float((q.abs() @ k.abs().T).max()) * scale
    return (d + 4) * SUM * most + 4 * SUM * (most + 10)


def attention_forward(q, k, v, cu, scale, causal, dtype):
    """(o, lse, bound of o, bound of lse) in 64 bits; rows outside the sequences are zero."""
    q, k, v = q.double(), k.double(), v.double()
    T, H, D = q.shape
    group = H // k.shape[1]
    o, ob = torch.zeros_like(q), torch.zeros_like(q)
    lse, lb = (torch.zeros(H, T, dtype=torch.float64, device=q.device) for _ in range(2))
    for a, b in spans(cu):
        if a == b:
            continue
        n = b - a
        for h in range(H):
            qs, ks, vs = q[a:b, h], k[a:b, h // group], v[a:b, h // group]
            s = _scores(qs, ks, scale, causal)
            lse[h, a:b] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[h, a:b, None])
            o[a:b, h] = p @ vs
            es = _score_error(qs, ks, scale)
            # every probability by its score, the exponential (2^-21) and, in bf16, its rounding; the row sum; the sum over the keys
            rel = 2 * es + 2.0 ** -20 + (u(dtype) if dtype != torch.float32 else 0.0) + 2 * (n + 4) * SUM
            ob[a:b, h] = (rel * p + TINY) @ vs.abs() + u(dtype) * o[a:b, h].abs() + TINY     # TINY: as in the backward pass below
            lb[h, a:b] = es + 2.0 ** -21 + (n + 4) * SUM + SUM * lse[h, a:b].abs()
    return o, lse, ob, lb


def attention_backward(q, k, v, o, lse, d_o, cu, scale, causal, dtype):
    """{name: (gradient, bound)} for the o and lse given."""
    q, k, v, o, lse, d_o = (x.double() for x in (q, k, v, o, lse, d_o))
    T, H, D = q.shape
    group = H // k.shape[1]
    g = {n: torch.zeros_like(x) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    e = {n: torch.zeros_like(x) for n, x in g.items()}
    low = u(dtype) if dtype != torch.float32 else 0.0
    for a, b in spans(cu):
        if a == b:
            continue
        n = b - a
        for h in range(H):
            kv = h // group
            qs, ks, vs, os, ds_o = q[a:b, h], k[a:b, kv], v[a:b, kv], o[a:b, h], d_o[a:b, h]
            p = torch.exp(_scores(qs, ks, scale, causal) - lse[h, a:b, None])
            row = (ds_o * os).sum(1, keepdim=True)
            ds = p * (ds_o @ vs.T - row)
            g["dq"][a:b, h] = scale * ds @ ks
            g["dk"][a:b, kv] += scale * ds.T @ qs
            g["dv"][a:b, kv] += p.T @ ds_o
            ep = 2 * _score_error(qs, ks, scale) + 2.0 ** -20
            # ds: its probability, the two inner products, its rounding to bf16; then the sums over rows or keys
            size = ds_o.abs() @ vs.abs().T + (ds_o * os).abs().sum(1, keepdim=True)
            # a probability below fp32's normal range may be zero, or any product with it: off by at most 2^-126 of the other factors
            eds = (ep + low + 4 * SUM) * ds.abs() + (p * (D + 2) * SUM + TINY) * size + TINY
            n_sum = group * n + 4
            e["dq"][a:b, h] += scale * (eds + (n + 4) * SUM * ds.abs()) @ ks.abs()
            e["dk"][a:b, kv] += scale * (eds + n_sum * SUM * ds.abs()).T @ qs.abs()
            e["dv"][a:b, kv] += ((ep + low + n_sum * SUM) * p.T + TINY) @ ds_o.abs() + TINY
    return {name: (g[name], e[name] + u(dtype) * g[name].abs()) for name in g}


def logprobs(x, targets, k):
    """{name: value} in 64 bits, for rows of every kind."""
    x = x.double()
    n, vocab = x.shape
    none = ~(x.amax(1) < math.inf) | x.isnan().any(1)
    empty = (x == -math.inf).all(1)
    safe = torch.where((none | empty)[:, None], 0.0, x)
    lse = torch.logsumexp(safe, 1)
    logp = torch.log_softmax(safe, 1)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    nan, ninf = math.nan, -math.inf

    def of(value, at_empty):
        shape = [n] + [1] * (value.dim() - 1)
        return torch.where(none.view(shape), nan, torch.where(empty.view(shape), at_empty, value))
    out = dict(lse=of(lse, ninf), entropy=of(entropy, 0.0))
    if targets is not None:
        y = targets.long()
        lp = of(logp.gather(1, y.clamp(0, vocab - 1)[:, None])[:, 0], ninf)
        out["logprob"] = torch.where(y < 0, 0.0, torch.where(y >= vocab, nan, lp))
    if k:
        order = torch.sort(torch.where(none[:, None], 0.0, x), dim=1, descending=True, stable=True).indices[:, :k]
        out["top_ids"] = torch.where(none[:, None], -1, order).to(torch.int32)
        out["top_logprob"] = of(logp.gather(1, order), ninf)
    return out


def logprobs_backward(x, targets, lse, entropy, gl, gh):
    """Gradient in 64 bits from the lse and entropy given, but for rows whose lse is too large (either gradient may be None)."""
    x, lse = x.double(), lse.double()
    n, vocab = x.shape
    empty = lse == -math.inf
    logp = x - torch.where(empty, 0.0, lse)[:, None]
    coarse = (lse.abs() > 4096) & ~empty                     # p from the logits themselves
    logp = torch.where(coarse[:, None], torch.log_softmax(torch.where(coarse[:, None], x, 0.0), 1), logp)
    p = logp.exp()
    dx = torch.zeros_like(x)
    if gl is not None:
        y = targets.long()
        g = torch.where(y < 0, 0.0, torch.where(y >= vocab, math.nan, gl.double()))
        dx -= g[:, None] * p
        dx[torch.arange(n, device=x.device), y.clamp(0, vocab - 1)] += g
    if gh is not None:
        dx -= gh.double()[:, None] * torch.where(p > 0, p * (logp + entropy.double()[:, None]), torch.where(p.isnan(), math.nan, 0.0))
    return torch.where(empty[:, None], 0.0, dx)


def clip(grads, max_norm):
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    scale = max_norm / total if math.isfinite(total) and total > max_norm else 1.0
    return total, scale
