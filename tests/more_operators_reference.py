"""Plain 64-bit forms of cross attention, head norms with rotation, dropout and the policy loss, with bounds on how far a correct
fp32 or bf16 implementation may be off (roundings counted as in operators_reference)."""
import math

import numpy as np
import torch

from operators_reference import SUM, TINY, U32, _score_error, spans, u


def cross_forward(q, k, v, cu, cu_kv, scale, dtype):
    """(o, lse, bound of o, bound of lse) in 64 bits; rows outside the sequences are zero, rows without keys have lse -infinity."""
    q, k, v = q.double(), k.double(), v.double()
    T, H, D = q.shape
    group = H // k.shape[1]
    o, ob = torch.zeros_like(q), torch.zeros_like(q)
    lse, lb = (torch.zeros(H, T, dtype=torch.float64, device=q.device) for _ in range(2))
    for (a, b), (x, y) in zip(spans(cu), spans(cu_kv)):
        if a == b:
            continue
        n = y - x
        if n == 0:
            lse[:, a:b] = -math.inf
            continue
        for h in range(H):
            qs, ks, vs = q[a:b, h], k[x:y, h // group], v[x:y, h // group]
            s = (qs @ ks.T) * scale
            lse[h, a:b] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[h, a:b, None])
            o[a:b, h] = p @ vs
            es = _score_error(qs, ks, scale)
            # as for attention over a sequence's own tokens: the score, the exponential (2^-21), its rounding in bf16, the two sums
            rel = 2 * es + 2.0 ** -20 + (u(dtype) if dtype != torch.float32 else 0.0) + 2 * (n + 4) * SUM
            ob[a:b, h] = (rel * p + TINY) @ vs.abs() + u(dtype) * o[a:b, h].abs() + TINY
            lb[h, a:b] = es + 2.0 ** -21 + (n + 4) * SUM + SUM * lse[h, a:b].abs()
    return o, lse, ob, lb


def cross_backward(q, k, v, o, lse, d_o, cu, cu_kv, scale, dtype):
    """{name: (gradient, bound)} for the o and lse given."""
    q, k, v, o, lse, d_o = (x.double() for x in (q, k, v, o, lse, d_o))
    T, H, D = q.shape
    group = H // k.shape[1]
    g = {n: torch.zeros_like(x) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    e = {n: torch.zeros_like(x) for n, x in g.items()}
    low = u(dtype) if dtype != torch.float32 else 0.0
    for (a, b), (x, y) in zip(spans(cu), spans(cu_kv)):
        if a == b or x == y:
            continue
        for h in range(H):
            kv = h // group
            qs, ks, vs, os, ds_o = q[a:b, h], k[x:y, kv], v[x:y, kv], o[a:b, h], d_o[a:b, h]
            p = torch.exp((qs @ ks.T) * scale - lse[h, a:b, None])
            ds = p * (ds_o @ vs.T - (ds_o * os).sum(1, keepdim=True))
            g["dq"][a:b, h] = scale * ds @ ks
            g["dk"][x:y, kv] += scale * ds.T @ qs
            g["dv"][x:y, kv] += p.T @ ds_o
            ep = 2 * _score_error(qs, ks, scale) + 2.0 ** -20
            size = ds_o.abs() @ vs.abs().T + (ds_o * os).abs().sum(1, keepdim=True)
            eds = (ep + low + 4 * SUM) * ds.abs() + (p * (D + 2) * SUM + TINY) * size + TINY
            n_sum = group * (b - a) + 4
            e["dq"][a:b, h] += scale * (eds + (y - x + 4) * SUM * ds.abs()) @ ks.abs()
            e["dk"][x:y, kv] += scale * (eds + n_sum * SUM * ds.abs()).T @ qs.abs()
            e["dv"][x:y, kv] += ((ep + low + n_sum * SUM) * p.T + TINY) @ ds_o.abs() + TINY
    return {name: (g[name], e[name] + u(dtype) * g[name].abs()) for name in g}
