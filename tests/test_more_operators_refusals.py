"""Calls of cross attention, head norms, dropout and the policy loss that are refused before anything reaches a GPU."""
import ctypes as C
import math
import random

import pytest
import torch

from paper_1910_05124_b200 import binding as B
from paper_1910_05124_b200 import build

P = 1 << 30           # addresses that are never followed


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def status(L, st):
    return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()


def at(i):
    return P + (i << 20)


def view(data, token=64, head=8):
    return C.byref(B.pm_head_view(data, token, head))


# ---- cross attention ------------------------------------------------------------------------------------------------

def cross_desc(**kw):
    d = dict(dtype=B.PM_F32, n_heads=4, n_kv_heads=2, head_dim=8, n_seqs=2, n_tokens=10, n_kv_tokens=20, scale=1.0)
    d.update(kw)
    return B.pm_cross_attention_desc(**d)


def cross(L, d, q=at(0), k=at(1), v=at(2), cu=at(3), cu_kv=at(4), o=at(5), lse=None):
    return status(L, L.pm_attention_cross_forward(C.byref(d), view(q), view(k), view(v), cu, cu_kv, view(o), lse, None))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), "PM_ERR_INVALID_ARG"), (dict(n_kv_heads=3), "PM_ERR_INVALID_ARG"), (dict(n_heads=0), "PM_ERR_INVALID_ARG"), (dict(head_dim=0), "PM_ERR_INVALID_ARG"),
    (dict(head_dim=129), "PM_ERR_UNSUPPORTED"), (dict(n_tokens=-1), "PM_ERR_INVALID_ARG"), (dict(n_kv_tokens=-1), "PM_ERR_INVALID_ARG"), (dict(n_seqs=-1), "PM_ERR_INVALID_ARG"),
    (dict(n_tokens=1 << 31), "PM_ERR_SHAPE"), (dict(n_kv_tokens=1 << 31), "PM_ERR_SHAPE"), (dict(n_seqs=(1 << 24) + 1), "PM_ERR_SHAPE"), (dict(scale=0.0), "PM_ERR_INVALID_ARG"),
    (dict(scale=math.nan), "PM_ERR_INVALID_ARG"), (dict(scale=math.inf), "PM_ERR_INVALID_ARG")])
def test_cross_descriptions(L, kw, code):
    assert cross(L, cross_desc(**kw))[0] == code
    assert status(L, L.pm_attention_cross_forward(None, *[None] * 6, None, None))[0] == "PM_ERR_INVALID_ARG"


def test_cross_pointers(L):
    d = cross_desc()
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(cu=None), dict(cu_kv=None), dict(q=at(0) + 2), dict(k=at(1) + 1)):
        assert cross(L, d, **kw)[0] == "PM_ERR_INVALID_ARG", kw
    # nothing to do: no pointer is looked at
    for kw in (dict(n_tokens=0), dict(n_seqs=0)):
        assert L.pm_attention_cross_forward(C.byref(cross_desc(**kw)), *[None] * 6, None, None) == 0
    # outputs that reach into an input, lse into o
    for kw in (dict(o=at(0)), dict(o=at(1) - 4 * (9 * 64 + 31)), dict(o=at(2) + 4 * (19 * 64 + 15)), dict(o=at(4) + 8 - 4 * 32), dict(o=at(3) - 4), dict(lse=at(5) + 4 * (64 * 9 + 31)),
               dict(lse=at(4)), dict(lse=at(0) - 156)):
        assert "output" in cross(L, d, **kw)[1] and cross(L, d, **kw)[0] == "PM_ERR_INVALID_ARG", kw


def test_cross_more_blocks_than_a_launch_has(L):
    far = 1 << 40
    for dtype in (B.PM_F32, B.PM_BF16):
        for dim in (64, 128):
            for tokens in (100, 1 << 14):                    # few query rows to a sequence, and more
                n_seqs = 1 << 24 if tokens == 100 else 1 << 17
                d = cross_desc(dtype=dtype, n_heads=65535, n_kv_heads=65535, head_dim=dim, n_seqs=n_seqs, n_tokens=tokens, n_kv_tokens=100)
                row = 65535 * dim
                st, msg = status(L, L.pm_attention_cross_forward(C.byref(d), view(far, row, dim), view(2 * far, row, dim), view(3 * far, row, dim), 4 * far, 5 * far, view(6 * far, row, dim), None, None))
                assert st == "PM_ERR_SHAPE" and "blocks" in msg, (st, msg)


def bytes_of(view, tokens, heads, dim, size):
    p, token, head = view
    return {p + (t * token + h * head) * size + b for t in range(tokens) for h in range(heads) for b in range(dim * size)}


@pytest.mark.parametrize("seed", range(4))
def test_cross_backward_views(L, seed):
    """Random layouts of the eight tensors, element by element.  Without a workspace a call whose tensors lie apart ends with PM_ERR_NOMEM."""
    rng, seen = random.Random(seed), {True: 0, False: 0}
    for _ in range(1000):
        dtype = rng.choice([B.PM_F32, B.PM_BF16])
        size = 4 if dtype == B.PM_F32 else 2
        n, m, K, dim = rng.randint(1, 5), rng.randint(1, 5), rng.randint(1, 3), rng.randint(1, 5)
        H = K * rng.randint(1, 2)
        kinds = [(n, H), (m, K), (m, K), (n, H), (n, H), (n, H), (m, K), (m, K)]             # q, k, v, o, d_o, dq, dk, dv
        views = []
        for i in range(8):
            near = P if rng.random() < 0.15 else P + (i << 16)
            views.append((near + size * rng.randint(0, 80), rng.randint(0, 60), rng.choice([dim, rng.randint(0, 20), rng.randint(0, 60)])))
        lse, cu, cu_kv = (P + (i << 16) if rng.random() < 0.8 else P + 4 * rng.randint(0, 100) for i in (20, 21, 22))
        sets = [bytes_of(v, t, h, dim, size) for v, (t, h) in zip(views, kinds)]
        reads = sets[:5] + [set(range(p, p + b)) for p, b in ((lse, 4 * H * n), (cu, 8), (cu_kv, 8))]
        overlap = any(w & r for w in sets[5:] for r in reads) or any(a & b for i, a in enumerate(sets[5:]) for b in sets[5:5 + i])
        d = B.pm_cross_attention_desc(dtype, H, K, dim, 1, n, m, 1.0)
        v = [view(*x) for x in views]
        st, msg = status(L, L.pm_attention_cross_backward(C.byref(d), *v[:4], lse, v[4], cu, cu_kv, *v[5:], None, 0, None))
        assert st == ("PM_ERR_INVALID_ARG" if overlap else "PM_ERR_NOMEM"), (views, msg)
        seen[overlap] += 1
    assert min(seen.values()) > 100, seen


def test_cross_backward_workspace(L):
    d = cross_desc()
    need = L.pm_attention_cross_workspace_bytes(C.byref(d))
    assert need == 4 * 4 * 10 and L.pm_attention_cross_workspace_bytes(None) == 0
    v = [view(at(i)) for i in range(8)]

    def call(lse=at(8), ws=at(11), n=need):
        return status(L, L.pm_attention_cross_backward(C.byref(d), *v[:4], lse, v[4], at(9), at(10), *v[5:], ws, n, None))
    assert call(lse=None)[0] == "PM_ERR_INVALID_ARG"
    assert call(ws=None)[0] == "PM_ERR_NOMEM" and str(need) in call(n=need - 1)[1]
    for ws in (at(11) + 2, at(0), at(8) + 156, at(10) + 8, at(7) - need + 4):
        assert call(ws=ws)[0] == "PM_ERR_INVALID_ARG", ws


# ---- head norms -----------------------------------------------------------------------------------------------------

TURNS = (C.c_uint64 * 64)()


def norm_desc(**kw):
    d = dict(dtype=B.PM_F32, n_heads=4, n_kv_heads=2, head_dim=8, rotary_dim=8, interleaved=0, n_tokens=10, eps=1e-6, turns=C.cast(TURNS, C.POINTER(C.c_uint64)))
    d.update(kw)
    return B.pm_head_norm_desc(**d)


def norm(L, d, q=at(0), k=at(1), pos=at(2), gq=at(3), gk=at(4), oq=at(5), ok=at(6), token=64):
    return status(L, L.pm_head_norm_rotate(C.byref(d), view(q, token), view(k, token), pos, gq, gk, view(oq, token), view(ok, token), None))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), "PM_ERR_INVALID_ARG"), (dict(head_dim=0), "PM_ERR_INVALID_ARG"), (dict(head_dim=129), "PM_ERR_UNSUPPORTED"), (dict(n_heads=-1), "PM_ERR_INVALID_ARG"),
    (dict(n_heads=0, n_kv_heads=0), "PM_ERR_INVALID_ARG"), (dict(n_heads=65536), "PM_ERR_SHAPE"), (dict(rotary_dim=10), "PM_ERR_INVALID_ARG"), (dict(rotary_dim=3), "PM_ERR_INVALID_ARG"),
    (dict(rotary_dim=-2), "PM_ERR_INVALID_ARG"), (dict(turns=None), "PM_ERR_INVALID_ARG"), (dict(n_tokens=-1), "PM_ERR_INVALID_ARG"), (dict(n_tokens=1 << 31), "PM_ERR_SHAPE"),
    (dict(eps=-1.0), "PM_ERR_INVALID_ARG"), (dict(eps=math.nan), "PM_ERR_INVALID_ARG"), (dict(eps=math.inf), "PM_ERR_INVALID_ARG"), (dict(n_tokens=0), "PM_OK")])
def test_norm_descriptions(L, kw, code):
    assert norm(L, norm_desc(**kw))[0] == code


def test_norm_pointers(L):
    d = norm_desc()
    assert L.pm_head_norm_rotate(None, *[None] * 8) == 1
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(gq=None), dict(gk=None), dict(oq=None), dict(ok=None), dict(q=at(0) + 2), dict(pos=at(2) + 2), dict(gq=at(3) + 1), dict(token=-1)):
        assert norm(L, d, **kw)[0] == "PM_ERR_INVALID_ARG", kw
    # other overlaps than an output that is its own input; those would be launched
    for kw in (dict(oq=at(0) + 4), dict(oq=at(1)), dict(ok=at(0)), dict(oq=at(2) + 36), dict(ok=at(3)), dict(oq=at(4) + 28), dict(oq=at(6)), dict(ok=at(5) + 4 * (9 * 64 + 31))):
        assert "overlap" in norm(L, d, **kw)[1], kw


def test_norm_backward(L):
    d = norm_desc()
    need = L.pm_head_norm_rotate_workspace_bytes(C.byref(d))
    assert need > 0 and L.pm_head_norm_rotate_workspace_bytes(None) == 0

    def call(d=d, dq=at(7), dk=at(8), dgq=at(9), dgk=at(10), ws=at(11), n=need, dyq=at(5), k=at(1)):
        return status(L, L.pm_head_norm_rotate_backward(C.byref(d), view(at(0)), view(k), at(2), at(3), at(4), view(dyq), view(at(6)), view(dq), view(dk), dgq, dgk, ws, n, None))
    assert call(ws=None)[0] == "PM_ERR_NOMEM" and str(need) in call(n=need - 1)[1]
    for kw in (dict(dq=None), dict(dk=None), dict(k=None), dict(dyq=None), dict(dgq=at(9) + 2), dict(ws=at(11) + 2), dict(d=norm_desc(n_kv_heads=0))):
        assert call(**kw)[0] == "PM_ERR_INVALID_ARG", kw
    for kw in (dict(dq=at(0)), dict(dq=at(5) + 4), dict(dq=at(6)), dict(dk=at(7)), dict(dgq=at(3)), dict(dgq=at(10) + 28), dict(dgk=at(2) + 36), dict(ws=at(0) - need + 4), dict(ws=at(9) + 28),
               dict(ws=at(8)), dict(dgq=at(7) + 4)):
        assert "overlap" in call(**kw)[1], kw


def test_rotation_turns(L):
    """Frequencies in 2^-64 turns: exact to half a unit, at every width."""
    from decimal import Decimal, getcontext
    getcontext().prec = 50
    turns = (C.c_uint64 * 64)()
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097")
    for rotary, base in ((2, 10000.0), (64, 10000.0), (128, 5e5), (80, 1.0), (128, 1e9)):
        assert L.pm_rotation_turns(rotary, base, turns) == 0
        for i in range(rotary // 2):
            want = (Decimal(base).ln() * (-2 * i) / rotary).exp() / (2 * pi) * 2 ** 64
            assert abs(turns[i] - want) <= 1 + want * Decimal(2) ** -60, (rotary, base, i)
    for bad in ((3, 10.0), (-2, 10.0), (130, 10.0), (8, 0.5), (8, math.nan), (8, math.inf)):
        assert L.pm_rotation_turns(*bad, turns) == 1
    assert L.pm_rotation_turns(8, 10.0, None) == 1


# ---- dropout --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "PM_ERR_INVALID_ARG"), (dict(n=-1), "PM_ERR_INVALID_ARG"), (dict(n=(1 << 42) + 1), "PM_ERR_SHAPE"), (dict(p=-0.1), "PM_ERR_INVALID_ARG"), (dict(p=1.0), "PM_ERR_INVALID_ARG"),
    (dict(p=1 - 2.0 ** -18), "PM_ERR_INVALID_ARG"), (dict(p=math.nan), "PM_ERR_INVALID_ARG"), (dict(x=None), "PM_ERR_INVALID_ARG"), (dict(y=None), "PM_ERR_INVALID_ARG"),
    (dict(rng=None), "PM_ERR_INVALID_ARG"), (dict(rng=at(2) + 4), "PM_ERR_INVALID_ARG"), (dict(x=at(0) + 2), "PM_ERR_INVALID_ARG"), (dict(res=at(1) + 1), "PM_ERR_INVALID_ARG"),
    (dict(y=at(0) + 4), "PM_ERR_INVALID_ARG"), (dict(y=at(1) - 396), "PM_ERR_INVALID_ARG"), (dict(y=at(2) + 12), "PM_ERR_INVALID_ARG"), (dict(y=at(2) - 396), "PM_ERR_INVALID_ARG"), (dict(n=0), "PM_OK")])
def test_dropout_arguments(L, kw, code):
    a = dict(x=at(0), res=at(1), dtype=B.PM_F32, n=100, p=0.1, rng=at(2), y=at(3))
    a.update(kw)
    assert status(L, L.pm_dropout(*a.values(), None))[0] == code
    if "res" not in kw and kw.get("y") != at(1) - 396:
        assert status(L, L.pm_dropout_backward(a["x"], a["dtype"], a["n"], a["p"], a["rng"], a["y"], None))[0] == code


# ---- policy loss ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,code", [
    (dict(low=-0.1), "PM_ERR_INVALID_ARG"), (dict(low=1.1), "PM_ERR_INVALID_ARG"), (dict(low=math.nan), "PM_ERR_INVALID_ARG"), (dict(high=-0.1), "PM_ERR_INVALID_ARG"),
    (dict(high=math.nan), "PM_ERR_INVALID_ARG"), (dict(kl=math.inf), "PM_ERR_INVALID_ARG"), (dict(ent=math.nan), "PM_ERR_INVALID_ARG"), (dict(ref=None), "PM_ERR_INVALID_ARG"),
    (dict(entropy=None), "PM_ERR_INVALID_ARG"), (dict(n=-1), "PM_ERR_INVALID_ARG"), (dict(n=(1 << 40) + 1), "PM_ERR_SHAPE"), (dict(lp=None), "PM_ERR_INVALID_ARG"),
    (dict(old=None), "PM_ERR_INVALID_ARG"), (dict(adv=None), "PM_ERR_INVALID_ARG"), (dict(stats=None), "PM_ERR_INVALID_ARG"), (dict(lp=at(0) + 2), "PM_ERR_INVALID_ARG"),
    (dict(d_lp=at(0)), "PM_ERR_INVALID_ARG"), (dict(d_ent=at(4) - 396), "PM_ERR_INVALID_ARG"), (dict(stats=at(5) + 396), "PM_ERR_INVALID_ARG"), (dict(d_lp=at(8)), "PM_ERR_INVALID_ARG"),
    (dict(stats=at(7) + 396), "PM_ERR_INVALID_ARG"), (dict(n=20000), "PM_ERR_NOMEM"), (dict(n=20000, ws=at(9), n_ws=1 << 19, lp=at(20)), "PM_ERR_NOMEM")])
def test_policy_arguments(L, kw, code):
    a = dict(low=0.2, high=0.2, kl=0.1, ent=0.1, mean=1, n=100, lp=at(0), old=at(1), adv=at(2), ref=at(3), entropy=at(4), w=at(5), stats=at(6), d_lp=at(7), d_ent=at(8), ws=None, n_ws=0)
    a.update(kw)
    if a["n_ws"]:
        a["n_ws"] = L.pm_policy_loss_workspace_bytes(a["n"]) - 1
    values = list(a.values())
    assert status(L, L.pm_policy_loss(C.byref(B.pm_policy_desc(*values[:5])), *values[5:], None))[0] == code


def test_policy_workspace(L):
    assert L.pm_policy_loss_workspace_bytes(16384) == 0
    need = L.pm_policy_loss_workspace_bytes(16385)
    d = B.pm_policy_desc(0.2, 0.2, 0.0, 0.0, 1)

    def call(ws):
        return status(L, L.pm_policy_loss(C.byref(d), 16385, at(0), at(1), at(2), None, None, at(3), at(4), at(5), None, ws, need, None))
    for ws in (at(6) + 4, at(0) + 16384 * 4, at(5) - need + 8, at(4) + 16):
        assert call(ws)[0] == "PM_ERR_INVALID_ARG", ws
    assert L.pm_policy_loss(None, *[0] + [None] * 9, None, 0, None) == 1


# ---- the classes ----------------------------------------------------------------------------------------------------

def test_python_checks(L):
    import paper_1910_05124_b200 as pm
    bad = [lambda: pm.CrossAttention(4, 3, 8), lambda: pm.CrossAttention(4, 2, 129), lambda: pm.CrossAttention(4, 2, 8, scale=0.0), lambda: pm.HeadNormRotate(0),
           lambda: pm.HeadNormRotate(129), lambda: pm.HeadNormRotate(7), lambda: pm.HeadNormRotate(8, rotary_dim=10), lambda: pm.HeadNormRotate(8, base=0.5), lambda: pm.HeadNormRotate(8, eps=-1.0),
           lambda: pm.Dropout(1.0), lambda: pm.Dropout(-0.1), lambda: pm.Dropout(math.nan), lambda: pm.PolicyLoss(clip_low=1.5), lambda: pm.PolicyLoss(clip_high=-1.0),
           lambda: pm.PolicyLoss(kl_coef=math.inf)]
    for make in bad:
        with pytest.raises(pm.PipeMareError):
            make()
    z = torch.zeros
    cpu = [lambda: pm.CrossAttention(4, 2, 8).pm_attention_cross_forward(z(3, 4, 8), z(3, 2, 8), z(3, 2, 8), z(2, dtype=torch.int32), z(2, dtype=torch.int32), z(3, 4, 8)),
           lambda: pm.HeadNormRotate(8).pm_head_norm_rotate(z(3, 4, 8), None, z(3, dtype=torch.int32), z(8), None, z(3, 4, 8), None),
           lambda: pm.Dropout(0.1).pm_dropout(z(3), z(2, dtype=torch.int64), z(3)), lambda: pm.PolicyLoss().pm_policy_loss(z(3), z(3), z(3), z(5))]
    for call in cpu:
        with pytest.raises(pm.PipeMareError, match="CUDA"):
            call()
    with pytest.raises(pm.PipeMareError, match="neither"):
        pm.HeadNormRotate(8).pm_head_norm_rotate(None, None, None, None, None, None, None)
    assert pm.Dropout.counters(0) == 0 and pm.Dropout.counters(1) == 1 and pm.Dropout.counters(17) == 3
