"""Which calls of the stand-alone operators are refused because a tensor that they write shares memory with another one.

No call here reaches a GPU: each lacks something that is checked after the overlap (a workspace, or one of its results)."""
import ctypes as C
import random

import pytest

from paper_1910_05124_b200 import binding as B
from paper_1910_05124_b200 import build

P = 1 << 30           # addresses that are never followed


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def bytes_of(view, tokens, heads, dim, size):
    at, token, head = view
    return {at + (t * token + h * head) * size + b for t in range(tokens) for h in range(heads) for b in range(dim * size)}


def attention_backward(L, views, tokens, H, K, dim, dtype, lse, cu, ws=None, n_ws=0):
    d = B.pm_attention_desc(dtype, H, K, dim, 1, 1, tokens, 1.0)
    v = [C.byref(B.pm_head_view(*x)) for x in views]
    st = L.pm_attention_packed_backward(C.byref(d), *v[:4], lse, v[4], cu, *v[5:], ws, n_ws, None)
    return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()


@pytest.mark.parametrize("seed", range(8))
def test_attention_backward_views(L, seed):
    """Random layouts of the eight tensors, element by element.  Without a workspace a call whose tensors lie apart ends with PM_ERR_NOMEM."""
    rng, seen = random.Random(seed), {True: 0, False: 0}
    for _ in range(1500):
        dtype = rng.choice([B.PM_F32, B.PM_BF16])
        size = 4 if dtype == B.PM_F32 else 2
        tokens, K, dim = rng.randint(1, 5), rng.randint(1, 3), rng.randint(1, 5)
        H = K * rng.randint(1, 2)
        heads = (H, K, K, H, H, H, K, K)
        views = []
        shared_token = rng.choice([None, rng.randint(1, 70)])
        for i, n in enumerate(heads):
            near = P if rng.random() < 0.15 else P + (i << 16)
            token = shared_token if shared_token and rng.random() < 0.8 else rng.randint(0, 60)
            views.append((near + size * rng.randint(0, 80), token, rng.choice([dim, rng.randint(0, 20), rng.randint(0, 60)])))
        lse = P + (20 << 16) if rng.random() < 0.8 else P + 4 * rng.randint(0, 100)
        cu = P + (21 << 16) if rng.random() < 0.8 else P + 4 * rng.randint(0, 100)
        sets = [bytes_of(v, tokens, n, dim, size) for v, n in zip(views, heads)]
        reads = sets[:5] + [set(range(lse, lse + 4 * H * tokens)), set(range(cu, cu + 8))]
        written = sets[5:]
        overlap = any(w & r for w in written for r in reads) or any(a & b for i, a in enumerate(written) for b in written[:i])
        status, message = attention_backward(L, views, tokens, H, K, dim, dtype, lse, cu)
        assert status == ("PM_ERR_INVALID_ARG" if overlap else "PM_ERR_NOMEM"), (views, tokens, H, K, dim, size, lse, cu, message)
        seen[overlap] += 1
    assert min(seen.values()) > 200, seen


def test_views_of_one_projection(L):
    """The gradients are slices of one buffer, heads in the last dimension or in front of the tokens; shifted by one they are refused."""
    T, H, K, D = 1000, 16, 4, 128
    row, size = (H + 2 * K) * D, 2
    inputs = [(P + (i << 26), H * D, D) for i in range(5)]
    far = dict(lse=P + (20 << 26), cu=P + (21 << 26))
    at = P + (8 << 26)

    def call(*outs):
        return attention_backward(L, inputs + list(outs), T, H, K, D, B.PM_BF16, **far)[0]
    assert call((at, row, D), (at + H * D * size, row, D), (at + (H + K) * D * size, row, D)) == "PM_ERR_NOMEM"
    for shift in (-size, size):
        assert call((at, row, D), (at + H * D * size + shift, row, D), (at + (H + K) * D * size, row, D)) == "PM_ERR_INVALID_ARG"
    first = (at, D, T * D), (at + H * T * D * size, D, T * D), (at + (H + K) * T * D * size, D, T * D)
    assert call(*first) == "PM_ERR_NOMEM"
    assert call(first[0], (first[1][0] - size, D, T * D), first[2]) == "PM_ERR_INVALID_ARG"
    # interleaved heads: every second one of a row, then the ones between
    even = (at, 2 * H * D, 2 * D), (at + D * size, 2 * H * D, 2 * D)
    assert call(even[0], even[1], (P + (9 << 26), K * D, D)) == "PM_ERR_NOMEM"
    T = 16                                                   # of different token strides, as many pairs as are looked at
    assert call(even[0], (even[1][0], 2 * H * D + 1, 2 * D), (P + (9 << 26), K * D, D)) == "PM_ERR_INVALID_ARG"
    T = 1000
    # an output that reaches into an input's last rows, without starting where it does
    assert call((inputs[3][0] + (T - 1) * H * D * size, H * D, D), (at, K * D, D), (P + (9 << 26), K * D, D)) == "PM_ERR_INVALID_ARG"


def test_attention_workspace(L):
    T, H, K, D = 100, 4, 2, 8
    views = [(P + (i << 20), n * D, D) for i, n in enumerate((H, K, K, H, H, H, K, K))]
    need = 4 * T * H
    for what in (views[0][0], views[3][0] + 32, views[7][0] - need + 4, P + (9 << 20) + need - 4):
        status, message = attention_backward(L, views, T, H, K, D, B.PM_F32, P + (9 << 20), P + (10 << 20), ws=what, n_ws=need)
        assert status == "PM_ERR_INVALID_ARG" and "workspace" in message, (what - P, message)


def test_attention_forward(L):
    T, H, K, D = 100, 4, 2, 8

    def call(o=P + (3 << 20), lse=P + (4 << 20), cu=P + (5 << 20)):
        d = B.pm_attention_desc(B.PM_F32, H, K, D, 1, 1, T, 1.0)
        v = [C.byref(B.pm_head_view(*x)) for x in ((P, H * D, D), (P + (1 << 20), K * D, D), (P + (2 << 20), K * D, D), (o, H * D, D))]
        st = L.pm_attention_packed_forward(C.byref(d), *v[:3], cu, v[3], lse, None)
        return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()
    for kw in (dict(o=P + 4), dict(o=P + (1 << 20) + 4 * (T * K * D - 1)), dict(o=P + (5 << 20) - 4 * T * H * D + 4), dict(lse=P + 400),
               dict(lse=P + (3 << 20) + 4), dict(lse=P + (5 << 20) + 4), dict(o=P + (2 << 20) - 4 * (T * H * D - 1))):
        status, message = call(**kw)
        assert status == "PM_ERR_INVALID_ARG" and "output" in message, (kw, message)


def logprobs(L, rows, vocab, stride, logits, targets, logprob, entropy, lse, k, top, ids):
    st = L.pm_token_logprobs(logits, B.PM_F32, rows, vocab, stride, targets, logprob, entropy, lse, k, top, ids, None)
    return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()


def test_logprob_results(L):
    rows, vocab, k = 10, 100, 4
    at = dict(logits=P, targets=P + (1 << 20), logprob=P + (2 << 20), entropy=P + (3 << 20), lse=P + (4 << 20), k=k, top=P + (5 << 20), ids=P + (6 << 20))
    for stride in (100, 108):
        for kw in (dict(logprob=P + 36), dict(entropy=P + 4 * 9 * stride + 396), dict(lse=P - 36), dict(top=P + 400 - 4), dict(ids=P + (1 << 20) + 36),
                   dict(entropy=P + (2 << 20) + 36), dict(lse=P + (5 << 20) + 4 * rows * k - 4), dict(logprob=P + (4 << 20) - 36), dict(ids=P + (5 << 20) + 4)):
            status, message = logprobs(L, rows, vocab, stride, **dict(at, **kw))
            assert status == "PM_ERR_INVALID_ARG" and ("share" in message or "overlaps" in message), (stride, kw, message)


def test_logprob_gradient(L):
    rows, vocab = 10, 100

    def call(d_logits, stride=100, grad_stride=100, lse=P + (1 << 20), **kw):
        a = dict(targets=P + (2 << 20), entropy=P + (3 << 20), d_logprob=P + (4 << 20), d_entropy=P + (5 << 20))
        a.update(kw)
        st = L.pm_token_logprobs_backward(P, B.PM_BF16, rows, vocab, stride, a["targets"], lse, a["entropy"], a["d_logprob"], a["d_entropy"], d_logits,
                                          grad_stride, None)
        return L.pm_status_string(st).decode(), L.pm_last_error(None).decode()
    far = P + (8 << 20)
    for a, kw in (((P + 2,), {}), ((P - 2,), {}), ((P + 2 * 999,), {}), ((P,), dict(grad_stride=108)), ((P + 198, 108, 108), {}), ((P + 200, 108, 100), {}),
                  ((far,), dict(lse=far + 1998)), ((far,), dict(targets=far - 36)), ((far, 108, 108), dict(d_logprob=far + 216 * 9 - 36)),
                  ((far,), dict(entropy=far + 400)), ((far,), dict(d_entropy=far + 4))):
        status, message = call(*a, **kw)
        assert status == "PM_ERR_INVALID_ARG" and "overlaps" in message, (a, kw, message)
