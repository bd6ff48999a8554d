"""Calls that the stand-alone operators refuse before anything reaches a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_1910_05124_b200 import binding as B
from paper_1910_05124_b200 import build


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def status(L, st):
    return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()


P = 1 << 20           # a pointer that is never followed: every call below is refused before a launch


def view(data=P, token=64, head=8):
    return C.byref(B.pm_head_view(data, token, head))


def attn(L, desc, *, q=None, cu=P, o=None):
    v = view()
    return L.pm_attention_packed_forward(C.byref(desc), q or v, v, v, cu, o or view(data=2 * P), None, None)


def desc(**kw):
    d = dict(dtype=B.PM_F32, n_heads=4, n_kv_heads=2, head_dim=8, n_seqs=2, causal=1, n_tokens=10, scale=1.0)
    d.update(kw)
    return B.pm_attention_desc(**d)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), "PM_ERR_INVALID_ARG"), (dict(n_kv_heads=3), "PM_ERR_INVALID_ARG"), (dict(n_heads=0), "PM_ERR_INVALID_ARG"),
    (dict(n_kv_heads=0), "PM_ERR_INVALID_ARG"), (dict(head_dim=0), "PM_ERR_INVALID_ARG"), (dict(head_dim=129), "PM_ERR_UNSUPPORTED"),
    (dict(n_tokens=-1), "PM_ERR_INVALID_ARG"), (dict(n_seqs=-1), "PM_ERR_INVALID_ARG"), (dict(n_tokens=1 << 31), "PM_ERR_SHAPE"),
    (dict(n_heads=1 << 17, n_kv_heads=1), "PM_ERR_SHAPE"), (dict(scale=0.0), "PM_ERR_INVALID_ARG"), (dict(scale=math.nan), "PM_ERR_INVALID_ARG"),
    (dict(scale=math.inf), "PM_ERR_INVALID_ARG"), (dict(scale=2.5e38), "PM_ERR_INVALID_ARG")])
def test_attention_descriptions(L, kw, code):
    assert status(L, attn(L, desc(**kw)))[0] == code


def test_attention_pointers(L):
    assert L.pm_attention_packed_forward(None, *[view()] * 3, P, view(), None, None) == 1
    assert attn(L, desc(), cu=None) == 1
    st, msg = status(L, attn(L, desc(), q=view(data=None)))
    assert st == "PM_ERR_INVALID_ARG" and "q" in msg
    assert status(L, attn(L, desc(), q=view(data=P + 2)))[0] == "PM_ERR_INVALID_ARG"       # fp32 at an odd half-word
    assert status(L, attn(L, desc(), q=view(token=-64)))[0] == "PM_ERR_INVALID_ARG"
    assert status(L, attn(L, desc(), o=view(data=None)))[0] == "PM_ERR_INVALID_ARG"
    st, msg = status(L, attn(L, desc(), o=view()))
    assert st == "PM_ERR_INVALID_ARG" and "output" in msg
    # nothing to do: no pointer is looked at
    assert L.pm_attention_packed_forward(C.byref(desc(n_tokens=0)), None, None, None, None, None, None, None) == 0
    assert L.pm_attention_packed_forward(C.byref(desc(n_seqs=0)), None, None, None, None, None, None, None) == 0


def test_attention_backward_workspace(L):
    d = desc()
    need = L.pm_attention_packed_workspace_bytes(C.byref(d))
    assert need >= 4 * 10 * 4
    assert L.pm_attention_packed_workspace_bytes(None) == 0
    v = [view()] * 4

    out = [view(data=i * P) for i in (2, 3, 4)]

    def call(lse=P, ws=P, n=need, out=out):
        return status(L, L.pm_attention_packed_backward(C.byref(d), *v, lse, view(), P, *out, ws, n, None))
    assert "input" in call(out=[view()] + out[1:])[1] and "same" in call(out=[out[0], out[1], out[0]])[1]
    assert call(lse=None)[0] == "PM_ERR_INVALID_ARG"
    assert call(ws=None)[0] == "PM_ERR_NOMEM"
    st, msg = call(n=need - 1)
    assert st == "PM_ERR_NOMEM" and str(need) in msg
    assert call(ws=P + 2)[0] == "PM_ERR_INVALID_ARG"


def lp(L, **kw):
    a = dict(logits=P, dtype=B.PM_F32, rows=3, vocab=10, stride=10, targets=P, logprob=P, entropy=None, lse=None, k=0, top=None, ids=None)
    a.update(kw)
    return status(L, L.pm_token_logprobs(*a.values(), None))[0]


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "PM_ERR_INVALID_ARG"), (dict(rows=-1), "PM_ERR_INVALID_ARG"), (dict(vocab=0), "PM_ERR_INVALID_ARG"),
    (dict(vocab=(1 << 24) + 1, stride=1 << 25), "PM_ERR_SHAPE"), (dict(rows=(1 << 24) + 1), "PM_ERR_SHAPE"), (dict(stride=9), "PM_ERR_INVALID_ARG"),
    (dict(logits=None), "PM_ERR_INVALID_ARG"), (dict(logits=P + 2), "PM_ERR_INVALID_ARG"), (dict(logprob=None), "PM_ERR_INVALID_ARG"),
    (dict(targets=None), "PM_ERR_INVALID_ARG"), (dict(k=11, top=P, ids=P), "PM_ERR_INVALID_ARG"), (dict(k=-1), "PM_ERR_INVALID_ARG"),
    (dict(vocab=100, stride=100, k=33, top=P, ids=P), "PM_ERR_INVALID_ARG"), (dict(k=2, ids=P), "PM_ERR_INVALID_ARG"), (dict(lse=P), "PM_ERR_INVALID_ARG"),
    (dict(entropy=2 * P, lse=2 * P), "PM_ERR_INVALID_ARG"), (dict(rows=0), "PM_OK")])
def test_logprob_arguments(L, kw, code):
    assert lp(L, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(gl=None), "PM_ERR_INVALID_ARG"), (dict(targets=None), "PM_ERR_INVALID_ARG"), (dict(gh=P), "PM_ERR_INVALID_ARG"),
    (dict(lse=None), "PM_ERR_INVALID_ARG"), (dict(grad=None), "PM_ERR_INVALID_ARG"), (dict(gstride=9), "PM_ERR_INVALID_ARG"), (dict(rows=0), "PM_OK")])
def test_logprob_backward_arguments(L, kw, code):
    a = dict(logits=P, dtype=B.PM_F32, rows=3, vocab=10, stride=10, targets=P, lse=P, entropy=None, gl=P, gh=None, grad=P, gstride=10)
    a.update(kw)
    assert status(L, L.pm_token_logprobs_backward(*a.values(), None))[0] == code


def test_clip_arguments(L):
    def call(pairs=((P, P, 4, 0, 0),), max_norm=1.0, norm=P, scale=P, ws=P, n_ws=1 << 20, n=None):
        arr = (B.pm_tensor_pair * max(1, len(pairs)))(*[B.pm_tensor_pair(*p) for p in pairs])
        return status(L, L.pm_clip_gradients(arr, len(pairs) if n is None else n, max_norm, norm, scale, ws, n_ws, None))[0]
    for kw in (dict(n=0), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(scale=None), dict(ws=P + 4),
               dict(pairs=((None, P, 4, 0, 0),)), dict(pairs=((P, None, 4, 0, 0),)), dict(pairs=((P, P, 4, 0, 2),)), dict(pairs=((P, P, 4, 0, 1),)),
               dict(pairs=((P + 2, P, 4, 0, 0),)), dict(pairs=((P, P + 1, 4, 1, 1),))):
        assert call(**kw) == "PM_ERR_INVALID_ARG", kw
    assert call(pairs=((P, P, 1 << 43, 0, 0),)) == "PM_ERR_SHAPE"
    assert call(pairs=((P, P, 1 << 42, 0, 0), (P, P, 1, 0, 0))) == "PM_ERR_SHAPE"
    need = L.pm_clip_gradients_workspace_bytes(1)
    assert call(ws=None) == "PM_ERR_NOMEM" and call(n_ws=need - 1) == "PM_ERR_NOMEM"
    assert L.pm_clip_gradients_workspace_bytes(0) == 0 and L.pm_clip_gradients_workspace_bytes(3000) > need


def test_python_checks_come_before_the_library(L):
    import paper_1910_05124_b200 as pm
    for bad in ((4, 3, 8), (0, 1, 8), (4, 2, 0), (4, 2, 129)):
        with pytest.raises(pm.PipeMareError):
            pm.PackedAttention(*bad)
    with pytest.raises(pm.PipeMareError):
        pm.PackedAttention(4, 2, 8, scale=0.0)
    with pytest.raises(pm.PipeMareError):
        pm.PackedAttention(4, 2, 8, scale=2.5e38)
    op = pm.PackedAttention(4, 2, 8)
    with pytest.raises(pm.PipeMareError, match="CUDA"):
        op.pm_attention_packed_forward(torch.zeros(3, 4, 8), torch.zeros(3, 2, 8), torch.zeros(3, 2, 8), torch.zeros(2, dtype=torch.int32),
                                       torch.zeros(3, 4, 8))
    for bad in (dict(vocab=0), dict(vocab=10, top_k=11), dict(vocab=100, top_k=33), dict(vocab=10, top_k=-1)):
        with pytest.raises(pm.PipeMareError):
            pm.TokenLogProbs(**bad)
    with pytest.raises(pm.PipeMareError, match="CUDA"):
        pm.TokenLogProbs(10).pm_token_logprobs(torch.zeros(2, 10), torch.zeros(2, dtype=torch.int32), torch.zeros(2))
    with pytest.raises(pm.PipeMareError, match="no tensors"):
        pm.GradClip([])
    with pytest.raises(pm.PipeMareError, match="CUDA"):
        pm.GradClip([torch.zeros(3)])


def test_overlapping_outputs_are_seen():
    """The rule on the strides of [tokens, heads, 8] outputs alone; it needs no memory."""
    import paper_1910_05124_b200 as pm
    op = pm.PackedAttention(4, 2, 8)
    good = [((3, 4, 8), (32, 8, 1)), ((3, 4, 8), (64, 16, 1)), ((3, 4, 8), (8, 24, 1)), ((1, 4, 8), (0, 8, 1))]
    bad = [((3, 4, 8), (0, 8, 1)), ((3, 4, 8), (32, 0, 1)), ((3, 4, 8), (31, 8, 1)), ((3, 4, 8), (8, 23, 1)), ((3, 4, 8), (32, 4, 1))]
    for shape, strides in good:
        op._check_apart("o", ((strides[0], shape[0]), (strides[1], shape[1])))
    for shape, strides in bad:
        with pytest.raises(pm.PipeMareError, match="overlaps"):
            op._check_apart("o", ((strides[0], shape[0]), (strides[1], shape[1])))
