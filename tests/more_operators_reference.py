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


# ---- norms and rotation ---------------------------------------------------------------------------------------------

PI = "3.14159265358979323846264338327950288419716939937510582097"


def rotation(positions, rotary, base):
    """cos, sin [tokens, rotary / 2] in 64 bits, from angles of 60 decimal digits taken into one turn."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    two_pi = 2 * Decimal(PI)
    freq = [(Decimal(base).ln() * (-2 * i) / rotary).exp() if i else Decimal(1) for i in range(rotary // 2)]
    angles = [[float((p * f) % two_pi) for f in freq] for p in positions.tolist()]
    a = torch.tensor(angles, dtype=torch.float64, device=positions.device).reshape(len(angles), rotary // 2)
    return a.cos(), a.sin()


def _pairs(rotary, interleaved):
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def _turn(x, cos, sin, a, b):
    """(turned, sum of the sizes that each result is made of)"""
    y, size = x.clone(), x.abs().clone()
    c, s = cos[:, None], sin[:, None]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


TRIG = 4 * U32        # of a sine or cosine: the angle's rounding (2.4e-8) and the function's two units in the last place


def norm_forward(x, gain, cos, sin, interleaved, eps, dtype):
    x, g = x.double(), gain.double()
    D = x.shape[-1]
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    y, size = _turn(x * r * g, cos, sin, *_pairs(2 * cos.shape[1], interleaved))
    # r: D squares summed, half of that error, its own two units; two products; a sine; two products and their sum
    rel = D * SUM / 2 + 8 * U32 + TRIG + 4 * U32
    return y, size * rel + u(dtype) * y.abs() + TINY


def norm_backward(x, gain, cos, sin, interleaved, eps, d_y, dtype):
    """(dx, its bound, d_gain, its bound)"""
    x, g, d_y = x.double(), gain.double(), d_y.double()
    D = x.shape[-1]
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    uu, size = _turn(d_y, cos, -sin, *_pairs(2 * cos.shape[1], interleaved))
    eu, er = size * (TRIG + 4 * U32), D * SUM / 2 + 4 * U32            # absolute error of u, relative error of r
    a, ea = g * uu, g.abs() * (eu + 2 * U32 * uu.abs())
    f = r * r * (a * x).mean(-1, keepdim=True)
    ef = r * r * ((ea * x.abs()).mean(-1, keepdim=True) + (a * x).abs().mean(-1, keepdim=True) * ((D + 6) * SUM + 2 * er))
    dx = r * (a - x * f)
    bound = r * (ea + x.abs() * ef + (a.abs() + (x * f).abs()) * (er + 6 * U32)) + u(dtype) * dx.abs() + TINY
    terms = uu * x * r
    n = x.shape[0] * x.shape[1]
    return dx, bound, terms.sum((0, 1)), (eu * (x * r).abs() + terms.abs() * (er + 4 * U32 + (n + 8) * SUM)).sum((0, 1)) + TINY


# ---- dropout --------------------------------------------------------------------------------------------------------

def philox(counters, key):
    """Philox4x32-10: uint32 [n, 4] of 128-bit counters (whole numbers), one Python integer at a time where the sums matter."""
    c = np.array([[n >> (32 * j) & 0xFFFFFFFF for j in range(4)] for n in counters], dtype=np.uint64)
    k0, k1, low, shift = key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF, np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[:, 0] * np.uint64(0xD2511F53), c[:, 2] * np.uint64(0xCD9E8D57)
        c = np.stack([(b >> shift) ^ c[:, 1] ^ np.uint64(k0), b & low, (a >> shift) ^ c[:, 3] ^ np.uint64(k1), a & low], axis=1)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c.astype(np.uint32)


def kept(n, p, seed, first):
    """Truth values of n elements and the scale."""
    words = philox([(first + i) % (1 << 64) for i in range(-(-n // 8))], seed % (1 << 64))
    bits = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(-1)[:n]
    dropped = int(p * 65536 + 0.5)
    return torch.from_numpy(bits >= dropped), 65536 / (65536 - dropped)


# ---- policy loss ----------------------------------------------------------------------------------------------------

def policy(lp, old, adv, ref, ent, weight, low, high, kl_coef, ent_coef, mean):
    """(stats, their bound, d_logprob, its bound, d_entropy) in 64 bits; tokens of weight 0 count for nothing."""
    w = torch.ones_like(lp, dtype=torch.float64) if weight is None else weight.double()
    live = w != 0

    def of(x):
        return torch.zeros_like(w) if x is None else torch.where(live, x.double(), 0.0)
    lp, old, adv, has_ref, ref, ent = of(lp), of(old), of(adv), ref is not None, of(ref), of(ent)
    total = w.sum()
    share = w / total if mean and float(total) else w * (0.0 if mean else 1.0)
    delta = lp - old
    ratio = delta.exp()
    clipped = ((delta > math.log1p(high)) & (adv > 0)) | ((delta < math.log1p(-low) if low < 1 else torch.zeros_like(live)) & (adv < 0))
    bound = (1.0 - low) + (delta > 0).double() * ((1.0 + high if math.isfinite(high) else 0.0) - (1.0 - low))
    pol = torch.where(adv == 0, 0.0, -torch.where(clipped, bound, ratio) * adv)
    free = torch.where(clipped | (adv == 0), 0.0, -ratio * adv)
    d = ref - lp if has_ref else torch.zeros_like(lp)
    kl, slope = torch.expm1(d) - d, torch.expm1(d)
    # of the ratio: the rounding of delta and the exponential's two units; of kl: the rounding of d, six units of the rest
    e_ratio = U32 * delta.abs() + 6 * U32
    e_kl, e_slope = slope.abs() * U32 * d.abs() + 8 * U32 * (kl + torch.where(d.abs() >= 0.5, slope.abs() + d.abs(), 0.0)), d.exp() * U32 * d.abs() + 4 * U32 * slope.abs()
    parts = [(share * pol).sum(), (share * kl).sum(), (share * ent).sum(), (share * clipped).sum()]
    errors = [(share * pol.abs() * e_ratio).sum(), (share * e_kl).sum(), 0.0, 0.0]
    loss = parts[0] + kl_coef * parts[1] - ent_coef * parts[2]
    stats = torch.stack([loss] + parts)
    e = [float(errors[0]) + kl_coef * float(errors[1])] + [float(x) for x in errors]
    e_stats = torch.tensor(e, dtype=torch.float64, device=lp.device) + 2 * U32 * stats.abs() + 1e-12 * float((share * (pol.abs() + ent.abs() + kl + 1)).sum())
    d_lp = share * (free - kl_coef * slope)
    e_lp = share * (free.abs() * (e_ratio + 4 * U32) + abs(kl_coef) * (e_slope + 4 * U32 * slope.abs())) + TINY
    return stats, e_stats + TINY, d_lp, e_lp, -ent_coef * share
