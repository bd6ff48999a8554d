"""Operators for programs with their own forward and backward pass, next to `FlatUpdate`: attention over packed sequences and over
those of another tensor, norms and rotation of queries and keys, dropout into a residual stream, log probabilities of given tokens,
the policy loss of sampled ones, and gradient clipping.  Argument checks and marshalling only; the tensors belong to the caller,
outputs included.

Every call is asynchronous on `stream` (default: the current stream of the tensors' device) and may be captured into a CUDA
graph.  As with any CUDA call, a tensor that another stream still writes has to be waited for by the caller, and a tensor
that belongs to another stream has to be kept until the call has run.  Refused arguments raise PipeMareError.
"""
import math
import struct
from bisect import bisect_left
from ctypes import addressof, byref, c_uint64

import torch

from .binding import PM_BF16, PM_F32, PipeMareError, _check, lib, pm_policy_desc, pm_tensor_pair

_DTYPES = {torch.float32: PM_F32, torch.bfloat16: PM_BF16}
_Tensor, _I32, _F32 = torch.Tensor, torch.int32, torch.float32
# pm_head_view and the descriptions as they lie in memory: what a call passes for a moment costs less as bytes than as ctypes objects
_VIEW, _ATTENTION, _CROSS, _HEAD_NORM = (struct.Struct(f).pack for f in ("@Pqq", "@6iqf4x", "@5iqqf4x", "@6iqfP"))


def _refuse(message, status="PM_ERR_INVALID_ARG"):
    raise PipeMareError(status, message)


def _mismatch(name, t, dtype, device, shape):
    """Refuses a tensor that is not of this type, device and shape."""
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} must be a tensor")
    if t.device != device:
        _refuse(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        _refuse(f"{name} is {t.dtype}, expected {dtype}")
    if tuple(t.shape) != shape:
        _refuse(f"{name} has shape {tuple(t.shape)}, expected {shape}", "PM_ERR_SHAPE")
    _refuse(f"{name} must be contiguous")


def _flat(name, t, dtype, device, shape):
    """Data pointer of a contiguous tensor; None for None."""
    if t is None:
        return None
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.get_device() == device.index and t.shape == shape and t.is_contiguous()):
        _mismatch(name, t, dtype, device, shape)
    return t.data_ptr()


def _flats(names, tensors, dtype, device, shape):
    """_flat of several tensors of one type and shape."""
    index, out = device.index, []
    for t in tensors:
        if t is None:
            out.append(None)
        elif isinstance(t, _Tensor) and t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
            out.append(t.data_ptr())
        else:
            _mismatch(names[len(out)], t, dtype, device, shape)
    return out


def _compute_device(name, t):
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        _refuse(f"{name} must be a CUDA tensor")
    if t.dtype not in _DTYPES:
        _refuse(f"{name} is {t.dtype}; float32 and bfloat16 are supported", "PM_ERR_UNSUPPORTED")
    return t.device


def _indexed(device):
    device = torch.device(device)
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


# the handle of the current stream without the object around it, where this torch has the call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(call, args, device, stream):
    """call(*args, stream handle) with the tensors' device current, and its status checked."""
    index = device.index
    if index != _current_device():
        with torch.cuda.device(device):
            return _launch(call, args, device, stream)
    if stream is None:
        status = call(*args, _raw_stream(index))
    else:
        if stream.device != device:
            _refuse(f"the stream belongs to {stream.device}, the tensors to {device}")
        status = call(*args, stream.cuda_stream)
    if status:
        _check(status)


def _launch_with(workspace, call, args, device, stream):
    """_launch of call(*args, workspace pointer, its bytes, stream handle).

    The workspace is device scratch of this call alone: it comes from the allocator's pool of the launching stream, so the
    memory is reused only by work queued behind the call (under capture it stays with the graph)."""
    if not workspace:
        return _launch(call, (*args, None, 0), device, stream)
    if device.index != _current_device():
        with torch.cuda.device(device):
            return _launch_with(workspace, call, args, device, stream)
    if stream is None or stream.cuda_stream == _raw_stream(device.index):
        scratch = torch.empty(workspace, dtype=torch.uint8, device=device)
    else:
        if stream.device != device:
            _refuse(f"the stream belongs to {stream.device}, the tensors to {device}")
        with torch.cuda.stream(stream):
            scratch = torch.empty(workspace, dtype=torch.uint8, device=device)
    _launch(call, (*args, scratch.data_ptr(), workspace), device, stream)


def _head_rows(name, t, heads, head_dim):
    """Device and number of tokens of a [tokens, heads, head_dim] tensor."""
    device = _compute_device(name, t)
    if t.dim() != 3:
        _refuse(f"{name} has shape {tuple(t.shape)}, expected [tokens, {heads}, {head_dim}]", "PM_ERR_SHAPE")
    return device, t.shape[0]


class _HeadTensors:
    """Views of [tokens, heads, head_dim] tensors, for classes with a head_dim."""

    def _views(self, shapes, dtype, device, names, tensors, n_read):
        """A pm_head_view for each of the tensors, of these shapes, checked; those behind the first n_read are written.  A shape of None gives
        None."""
        index, views = device.index, []
        for t, shape in zip(tensors, shapes):
            if shape is None:
                views.append(None)
                continue
            if not (isinstance(t, _Tensor) and t.dtype is dtype and t.get_device() == index and t.shape == shape):
                _mismatch(names[len(views)], t, dtype, device, shape)
            tokens, h, d = shape
            token, head, one = t.stride()
            if one != 1 and d > 1:
                _refuse(f"the last dimension of {names[len(views)]} must be contiguous")
            if (head != d or token < h * d) and len(views) >= n_read:
                self._check_apart(names[len(views)], ((token, tokens), (head, h)))
            views.append(_VIEW(t.data_ptr(), token, head))
        return views

    def _check_apart(self, name, dims):
        """Rows of one head, or heads of one row, of a tensor that is written must not share elements."""
        if min(n for _, n in dims) < 1:
            return
        end = self.head_dim
        for stride, n in sorted((s, n) for s, n in dims if n > 1):
            if stride < end:
                _refuse(f"{name} overlaps itself")
            end += stride * (n - 1)


class _HeadAttention(_HeadTensors):
    """What the attention classes share."""

    def __init__(self, n_heads, n_kv_heads, head_dim, scale):
        if n_heads < 1 or n_kv_heads < 1 or n_heads % n_kv_heads:
            _refuse("n_heads must be a positive multiple of n_kv_heads")
        if head_dim < 1:
            _refuse("head_dim must be positive")
        if head_dim > 128:
            _refuse("heads wider than 128", "PM_ERR_UNSUPPORTED")
        scale = head_dim ** -0.5 if scale is None else float(scale)
        if not 0 < scale < 2e38:
            _refuse("scale must be positive and below 2e38")
        self.n_heads, self.n_kv_heads, self.head_dim, self.scale = n_heads, n_kv_heads, head_dim, scale
        self.L = lib()

    def _starts(self, name, cu, device):
        """Pointer and number of sequences of an array of starts."""
        if not isinstance(cu, _Tensor) or cu.dim() != 1 or not (n := cu.numel()):
            _refuse(f"{name} must be a one-dimensional tensor of sequences + 1 entries", "PM_ERR_SHAPE")
        if not (cu.dtype is _I32 and cu.get_device() == device.index and cu.is_contiguous()):
            _mismatch(name, cu, _I32, device, (n,))
        return cu.data_ptr(), n - 1

    def pm_attention_packed_status(self, device="cuda", stream=None):
        """Raises if a device-side wait of a tensor-core kernel ran out since the last call on this device (a defect); synchronises
        the stream."""
        _launch(self.L.pm_attention_packed_status, (), _indexed(device), stream)

    def pm_attention_packed_selftest_wait_timeout(self, limit_cycles, device="cuda", stream=None):
        """Enqueues a wait that runs out after limit_cycles: the next pm_attention_packed_status on this device raises."""
        _launch(self.L.pm_attention_packed_selftest_wait_timeout, (int(limit_cycles),), _indexed(device), stream)


class PackedAttention(_HeadAttention):
    """Attention over sequences of different lengths laid end to end, with shared key/value heads.

    q, o: [tokens, n_heads, head_dim]; k, v: [tokens, n_kv_heads, head_dim]; all float32 or all bfloat16, the last dimension
    contiguous, the others at any stride (q, k and v may be views of one projection's output).  cu_seqlens: int32
    [sequences + 1] on the device, ascending; sequence b is tokens cu_seqlens[b] to cu_seqlens[b + 1] - 1, and tokens outside
    all sequences are neither used nor written.  lse: float32 [n_heads, tokens].  head_dim up to 128.
    """

    def __init__(self, n_heads, n_kv_heads, head_dim, *, causal=True, scale=None):
        super().__init__(n_heads, n_kv_heads, head_dim, scale)
        self.causal = bool(causal)

    def _desc(self, q, cu_seqlens):
        device, tokens = _head_rows("q", q, self.n_heads, self.head_dim)
        cu, n_seqs = self._starts("cu_seqlens", cu_seqlens, device)
        return device, (tokens, self.n_heads, self.head_dim), (tokens, self.n_kv_heads, self.head_dim), _ATTENTION(
            _DTYPES[q.dtype], self.n_heads, self.n_kv_heads, self.head_dim, n_seqs, self.causal, tokens, self.scale), cu

    def pm_attention_packed_forward(self, q, k, v, cu_seqlens, o, lse=None, stream=None):
        """Writes o and, for a backward pass, lse."""
        device, Q, K, desc, cu = self._desc(q, cu_seqlens)
        vq, vk, vv, vo = self._views((Q, K, K, Q), q.dtype, device, ("q", "k", "v", "o"), (q, k, v, o), 3)
        p_lse = _flat("lse", lse, _F32, device, (self.n_heads, Q[0]))
        _launch(self.L.pm_attention_packed_forward, (desc, vq, vk, vv, cu, vo, p_lse), device, stream)

    def pm_attention_packed_backward(self, q, k, v, o, lse, d_o, cu_seqlens, dq, dk, dv, stream=None):
        """Writes dq, dk and dv from d_o and what the forward call wrote."""
        device, Q, K, desc, cu = self._desc(q, cu_seqlens)
        if lse is None:
            _refuse("lse must be a tensor")
        vq, vk, vv, vo, vdo, *grads = self._views((Q, K, K, Q, Q, Q, K, K), q.dtype, device, ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"),
                                                  (q, k, v, o, d_o, dq, dk, dv), 5)
        p_lse = _flat("lse", lse, _F32, device, (self.n_heads, Q[0]))
        _launch_with(4 * self.n_heads * Q[0], self.L.pm_attention_packed_backward, (desc, vq, vk, vv, vo, p_lse, vdo, cu, *grads), device, stream)


class CrossAttention(_HeadAttention):
    """Attention of packed sequences over the sequences of another tensor, such as a decoder's tokens over an encoder's states.

    q, o: [tokens, n_heads, head_dim] with cu_seqlens; k, v: [kv_tokens, n_kv_heads, head_dim] with cu_seqlens_kv; the rest as in
    PackedAttention, without a causal mask.  Sequence b of q attends to every row of sequence b of k and v; without keys its o is
    zero and its lse -infinity.  A decoding step is a call with one token, or the few of a beam, to each sequence.
    """

    def __init__(self, n_heads, n_kv_heads, head_dim, *, scale=None):
        super().__init__(n_heads, n_kv_heads, head_dim, scale)

    def _desc(self, q, k, cu_seqlens, cu_seqlens_kv):
        device, tokens = _head_rows("q", q, self.n_heads, self.head_dim)
        kv_tokens = k.shape[0] if isinstance(k, _Tensor) and k.dim() else 0           # k's type and shape: with the others
        cu, n_seqs = self._starts("cu_seqlens", cu_seqlens, device)
        cu_kv, n_kv_seqs = self._starts("cu_seqlens_kv", cu_seqlens_kv, device)
        if n_seqs != n_kv_seqs:
            _refuse(f"cu_seqlens has {n_seqs} sequences, cu_seqlens_kv {n_kv_seqs}", "PM_ERR_SHAPE")
        return device, (tokens, self.n_heads, self.head_dim), (kv_tokens, self.n_kv_heads, self.head_dim), _CROSS(
            _DTYPES[q.dtype], self.n_heads, self.n_kv_heads, self.head_dim, n_seqs, tokens, kv_tokens, self.scale), cu, cu_kv

    def pm_attention_cross_forward(self, q, k, v, cu_seqlens, cu_seqlens_kv, o, lse=None, stream=None):
        """Writes o and, for a backward pass, lse."""
        device, Q, K, desc, cu, cu_kv = self._desc(q, k, cu_seqlens, cu_seqlens_kv)
        vq, vk, vv, vo = self._views((Q, K, K, Q), q.dtype, device, ("q", "k", "v", "o"), (q, k, v, o), 3)
        p_lse = _flat("lse", lse, _F32, device, (self.n_heads, Q[0]))
        _launch(self.L.pm_attention_cross_forward, (desc, vq, vk, vv, cu, cu_kv, vo, p_lse), device, stream)

    def pm_attention_cross_backward(self, q, k, v, o, lse, d_o, cu_seqlens, cu_seqlens_kv, dq, dk, dv, stream=None):
        """Writes dq, dk and dv from d_o and what the forward call wrote."""
        device, Q, K, desc, cu, cu_kv = self._desc(q, k, cu_seqlens, cu_seqlens_kv)
        if lse is None:
            _refuse("lse must be a tensor")
        vq, vk, vv, vo, vdo, *grads = self._views((Q, K, K, Q, Q, Q, K, K), q.dtype, device, ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"),
                                                  (q, k, v, o, d_o, dq, dk, dv), 5)
        p_lse = _flat("lse", lse, _F32, device, (self.n_heads, Q[0]))
        _launch_with(4 * self.n_heads * Q[0], self.L.pm_attention_cross_backward, (desc, vq, vk, vv, vo, p_lse, vdo, cu, cu_kv, *grads), device, stream)


class HeadNormRotate(_HeadTensors):
    """Root-mean-square norms of queries and keys for each head, with a gain, and the rotation of their first rotary_dim dimensions (None:
    all, 0: none) by the positions, in one pass.

    q, q_out: [tokens, n_heads, head_dim]; k, k_out: [tokens, n_kv_heads, head_dim]; all float32 or all bfloat16, at any strides with the
    last dimension contiguous; either side may be None with its gain and output.  positions: int32 [tokens] on the device (None
    without rotation).  gains: float32 [head_dim].  Pairs are (i, i + rotary_dim / 2) or, interleaved, (2 i, 2 i + 1); pair i turns by
    base^(-2 i / rotary_dim) a position, exactly at every position.
    """

    def __init__(self, head_dim, *, rotary_dim=None, base=10000.0, interleaved=False, eps=1e-6):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if head_dim < 1:
            _refuse("head_dim must be positive")
        if head_dim > 128:
            _refuse("heads wider than 128", "PM_ERR_UNSUPPORTED")
        if not 0 <= rotary_dim <= head_dim or rotary_dim % 2:
            _refuse("rotary_dim must be even and at most head_dim")
        if not 0 <= float(eps) <= 1e30:
            _refuse("eps must not be negative")
        self.head_dim, self.rotary_dim, self.base, self.interleaved, self.eps = head_dim, rotary_dim, float(base), bool(interleaved), float(eps)
        self.L = lib()
        self.turns = (c_uint64 * max(1, rotary_dim // 2))()
        _check(self.L.pm_rotation_turns(rotary_dim, self.base, self.turns))
        self.p_turns = addressof(self.turns)
        self.ws_bytes = self.L.pm_head_norm_rotate_workspace_bytes(_HEAD_NORM(PM_F32, 1, 1, head_dim, rotary_dim, 0, 0, 0.0, self.p_turns))

    def _sides(self, q, k, positions, q_gain, k_gain):
        """Device, dtype, shapes of both sides (None: absent), description, and pointers of positions and gains."""
        d, Q, K, p_q, p_k = self.head_dim, None, None, None, None
        lead, name = (q, "q") if q is not None else (k, "k")
        if lead is None:
            _refuse("neither queries nor keys")
        device, tokens = _head_rows(name, lead, "heads", d)
        if q is not None:
            if q.shape[1] < 1:
                _refuse("q has no heads", "PM_ERR_SHAPE")
            Q = tokens, q.shape[1], d
            p_q = _flat("q_gain", q_gain, _F32, device, (d,))
        if k is not None:
            if not isinstance(k, _Tensor) or k.dim() != 3 or k.shape[1] < 1:
                _refuse(f"k must be a tensor of [tokens, heads, {d}]", "PM_ERR_SHAPE")
            K = tokens, k.shape[1], d
            p_k = _flat("k_gain", k_gain, _F32, device, (d,))
        at = _flat("positions", positions, _I32, device, (tokens,)) if self.rotary_dim else None
        if self.rotary_dim and positions is None or Q and q_gain is None or K and k_gain is None:
            _refuse("positions must be a tensor" if self.rotary_dim and positions is None else "the gains must be tensors")
        desc = _HEAD_NORM(_DTYPES[lead.dtype], Q[1] if Q else 0, K[1] if K else 0, d, self.rotary_dim, self.interleaved, tokens, self.eps, self.p_turns)
        return device, lead.dtype, Q, K, desc, at, (p_q, p_k)

    def pm_head_norm_rotate(self, q, k, positions, q_gain, k_gain, q_out, k_out, stream=None):
        """Writes q_out and k_out, which may be q and k."""
        device, dtype, Q, K, desc, pos, gains = self._sides(q, k, positions, q_gain, k_gain)
        vq, vk, *outs = self._views((Q, K, Q, K), dtype, device, ("q", "k", "q_out", "k_out"), (q, k, q_out, k_out), 2)
        _launch(self.L.pm_head_norm_rotate, (desc, vq, vk, pos, *gains, *outs), device, stream)

    def pm_head_norm_rotate_backward(self, q, k, positions, q_gain, k_gain, d_q_out, d_k_out, dq, dk, d_q_gain=None, d_k_gain=None, stream=None):
        """Writes dq and dk (which may be d_q_out and d_k_out) and the gains' gradients that are given."""
        device, dtype, Q, K, desc, pos, gains = self._sides(q, k, positions, q_gain, k_gain)
        vq, vk, *views = self._views((Q, K, Q, K, Q, K), dtype, device, ("q", "k", "d_q_out", "d_k_out", "dq", "dk"), (q, k, d_q_out, d_k_out, dq, dk), 4)
        grads = _flats(("d_q_gain", "d_k_gain"), (d_q_gain, d_k_gain), torch.float32, device, (self.head_dim,))
        _launch_with(0 if d_q_gain is None and d_k_gain is None else self.ws_bytes, self.L.pm_head_norm_rotate_backward,
                     (desc, vq, vk, pos, *gains, *views, *grads), device, stream)


class Dropout:
    """Dropout with a mask that is never stored: formed from a counter-based generator in the forward and in the backward call.

    x, y, residual: tensors of one shape, contiguous, all float32 or all bfloat16.  rng: int64 [2] on the device, the generator's key and
    the first counter of this call, which uses counters(x.numel()) of them; the backward call takes the same two numbers.  They are
    read when the call runs: between replays of a captured graph the program moves the counter on.  p is taken to the nearest
    2^-16; what is kept is scaled by 1 / (1 - p).
    """

    def __init__(self, p):
        p = float(p)
        if not 0 <= p < 1 - 2.0 ** -17:
            _refuse("p must be 0 to below 1 - 2^-17")
        self.p = p
        self.L = lib()

    @staticmethod
    def counters(n):
        """How many counters a call on n elements uses."""
        return (n + 7) // 8

    def _tensors(self, names, tensors, rng):
        lead = tensors[0]
        device = _compute_device(names[0], lead)
        pointers = _flats(names, tensors, lead.dtype, device, lead.shape)
        if rng is None:
            _refuse("rng must be a tensor")
        return device, _DTYPES[lead.dtype], lead.numel(), pointers, _flat("rng", rng, torch.int64, device, (2,))

    def pm_dropout(self, x, rng, y, residual=None, stream=None):
        """Writes y (which may be x or the residual): what is kept of x, scaled, added to the residual."""
        device, dtype, n, (p_x, p_y, p_res), p_rng = self._tensors(("x", "y", "residual"), (x, y, residual), rng)
        if y is None:
            _refuse("y must be a tensor")
        _launch(self.L.pm_dropout, (p_x, p_res, dtype, n, self.p, p_rng, p_y), device, stream)

    def pm_dropout_backward(self, d_y, rng, d_x, stream=None):
        """Writes d_x (which may be d_y); the residual's gradient is d_y itself."""
        device, dtype, n, (p_y, p_x), p_rng = self._tensors(("d_y", "d_x"), (d_y, d_x), rng)
        if d_x is None:
            _refuse("d_x must be a tensor")
        _launch(self.L.pm_dropout_backward, (p_y, dtype, n, self.p, p_rng, p_x), device, stream)


class TokenLogProbs:
    """Log probabilities of given tokens under rows of logits [rows, vocab] (float32 or bfloat16, contiguous rows at any stride),
    the entropy of each row, its logsumexp, and its top_k most likely tokens.

    targets: int32 [rows], negative = padding.  logprob, entropy, lse: float32 [rows]; top_logprob: float32 [rows, top_k];
    top_ids: int32 [rows, top_k], equal logits in ascending order of their ids.
    """

    def __init__(self, vocab, top_k=0):
        if vocab < 1 or vocab > 1 << 24:
            _refuse("vocab must be 1 to 2^24")
        if not 0 <= top_k <= min(32, vocab):
            _refuse("top_k must be 0 to 32 and at most the vocabulary size")
        self.vocab, self.top_k = vocab, top_k
        self.L = lib()

    def _rows(self, name, t, like=None):
        device = _compute_device(name, t)
        if like is not None and not (t.dtype is like.dtype and t.device == like.device and t.shape == like.shape):
            _mismatch(name, t, like.dtype, like.device, tuple(like.shape))
        if t.dim() != 2 or t.shape[1] != self.vocab:
            _refuse(f"{name} has shape {tuple(t.shape)}, expected [rows, {self.vocab}]", "PM_ERR_SHAPE")
        stride, one = t.stride()
        if one != 1 and self.vocab > 1:
            _refuse(f"the rows of {name} must be contiguous")
        if t.shape[0] < 2:
            stride = self.vocab
        if stride < self.vocab:
            _refuse(f"the rows of {name} overlap")
        return device, stride

    def pm_token_logprobs(self, logits, targets, logprob, entropy=None, lse=None, top_logprob=None, top_ids=None, stream=None):
        """Writes logprob (targets and logprob may both be None) and whichever of the others are given."""
        device, stride = self._rows("logits", logits)
        n, k, f32, i32 = logits.shape[0], self.top_k, torch.float32, torch.int32
        if k and (top_logprob is None or top_ids is None):
            _refuse("top_logprob and top_ids must be given with top_k")
        args = (logits.data_ptr(), _DTYPES[logits.dtype], n, self.vocab, stride, _flat("targets", targets, i32, device, (n,)),
                _flat("logprob", logprob, f32, device, (n,)), _flat("entropy", entropy, f32, device, (n,)), _flat("lse", lse, f32, device, (n,)),
                k, _flat("top_logprob", top_logprob, f32, device, (n, k)), _flat("top_ids", top_ids, i32, device, (n, k)))
        _launch(self.L.pm_token_logprobs, args, device, stream)

    def pm_token_logprobs_backward(self, logits, targets, lse, d_logits, d_logprob=None, entropy=None, d_entropy=None, stream=None):
        """Writes d_logits (logits itself is allowed) from the gradients of logprob and / or of the entropy."""
        device, stride = self._rows("logits", logits)
        _, grad_stride = self._rows("d_logits", d_logits, logits)
        n, f32 = logits.shape[0], torch.float32
        if lse is None:
            _refuse("lse must be a tensor")
        if logits.data_ptr() == d_logits.data_ptr() and stride != grad_stride:
            _refuse("d_logits shares the memory of logits at other strides")
        args = (logits.data_ptr(), _DTYPES[logits.dtype], n, self.vocab, stride, _flat("targets", targets, torch.int32, device, (n,)),
                _flat("lse", lse, f32, device, (n,)), _flat("entropy", entropy, f32, device, (n,)),
                _flat("d_logprob", d_logprob, f32, device, (n,)), _flat("d_entropy", d_entropy, f32, device, (n,)),
                d_logits.data_ptr(), grad_stride)
        _launch(self.L.pm_token_logprobs_backward, args, device, stream)


class PolicyLoss:
    """Clipped policy loss of sampled tokens with a KL term to a reference and an entropy bonus, with its gradients, between
    TokenLogProbs' forward and backward call.

    All tensors float32 [tokens], contiguous: logprob, old_logprob, advantage; ref_logprob (needed with kl_coef) and entropy (needed with
    entropy_coef); weight (None: 1), 0 for padding, whose values count for nothing.  With mean the weights are divided by their sum, else
    they are taken as they are (1 / the tokens of all microbatches, say).  stats: float32 [5], the loss and the weighted sums of its
    policy term, of the KL term, of the entropy, and of the clipped tokens.
    """

    def __init__(self, *, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, mean=True):
        clip_low, clip_high, kl_coef, entropy_coef = float(clip_low), float(clip_high), float(kl_coef), float(entropy_coef)
        if not 0 <= clip_low <= 1:
            _refuse("clip_low must be 0 to 1")
        if not clip_high >= 0:
            _refuse("clip_high must not be negative")
        if not (math.isfinite(kl_coef) and math.isfinite(entropy_coef)):
            _refuse("coefficients must be finite")
        self.kl_coef, self.entropy_coef = kl_coef, entropy_coef
        self.desc = byref(pm_policy_desc(clip_low, clip_high, kl_coef, entropy_coef, bool(mean)))
        self.L = lib()

    def pm_policy_loss(self, logprob, old_logprob, advantage, stats, d_logprob=None, ref_logprob=None, entropy=None, d_entropy=None, weight=None,
                       stream=None):
        """Writes stats and the gradients that are given."""
        if not (isinstance(logprob, torch.Tensor) and logprob.is_cuda):
            _refuse("logprob must be a CUDA tensor")
        device, f32, n = logprob.device, torch.float32, logprob.numel()
        if old_logprob is None or advantage is None or stats is None:
            _refuse("old_logprob, advantage and stats must be tensors")
        if self.kl_coef and ref_logprob is None or self.entropy_coef and entropy is None:
            _refuse("kl_coef without ref_logprob" if self.kl_coef and ref_logprob is None else "entropy_coef without entropy")
        *ins, p_lp, p_ent = _flats(("logprob", "old_logprob", "advantage", "ref_logprob", "entropy", "weight", "d_logprob", "d_entropy"),
                                   (logprob, old_logprob, advantage, ref_logprob, entropy, weight, d_logprob, d_entropy), f32, device, (n,))
        _launch_with(self.L.pm_policy_loss_workspace_bytes(n), self.L.pm_policy_loss,
                     (self.desc, n, *ins, _flat("stats", stats, f32, device, (5,)), p_lp, p_ent), device, stream)


class GradClip:
    """Clipping of a list of gradient tensors by their global norm, into `outs` (None: in place).

    Holds the two lists (and so the tensors' memory) for calls to come; a program whose gradients move to other tensors makes a new one.
    Tensors are contiguous, float32 or bfloat16 in any mixture, on one device; outs[i] has as many elements as grads[i] and may be a
    slice of the gradient arena.
    """

    def __init__(self, grads, outs=None):
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if not grads:
            _refuse("no tensors")
        if len(outs) != len(grads):
            _refuse(f"{len(grads)} gradients, {len(outs)} destinations")
        self.device = _compute_device("grads[0]", grads[0])
        self.L = lib()
        self.grads, self.outs = grads, outs
        rows, spans = [], []
        for i, (g, o) in enumerate(zip(grads, outs)):
            if not (self._fits(g) and self._fits(o) and g.numel() == o.numel()):
                self._mismatch(i, g, o)
            n, src, dst, src_type, dst_type = g.numel(), g.data_ptr(), o.data_ptr(), _DTYPES[g.dtype], _DTYPES[o.dtype]
            rows.append((src, dst, n, src_type, dst_type))
            if n:
                spans.append((dst, dst + n * o.element_size(), True, i))
                if src != dst or src_type != dst_type:
                    spans.append((src, src + n * g.element_size(), False, i))
        self.tensors = (pm_tensor_pair * len(rows))(*rows)
        end = {True: (0, 0), False: (0, 0)}                  # the furthest end so far of what is written, and of what is read
        self.starts, self.stops = starts, stops = [], []     # of what the tensors cover, ascending
        for start, stop, written, i in sorted(spans):
            for other in (True, False) if written else (True,):
                if start < end[other][0]:
                    _refuse(f"{'outs' if written else 'grads'}[{i}] overlaps {'outs' if other else 'grads'}[{end[other][1]}]")
            if stop > end[written][0]:
                end[written] = (stop, i)
            starts.append(start)
            stops.append(max(stop, stops[-1]) if stops else stop)
        self.ws_bytes = self.L.pm_clip_gradients_workspace_bytes(len(grads))

    def _fits(self, t):
        return isinstance(t, torch.Tensor) and t.device == self.device and t.dtype in _DTYPES and t.is_contiguous()

    def _mismatch(self, i, g, o):
        for name, t in ((f"grads[{i}]", g), (f"outs[{i}]", o)):
            if _compute_device(name, t) != self.device:
                _refuse(f"{name} is on {t.device}, expected {self.device}")
            if not t.is_contiguous():
                _refuse(f"{name} must be contiguous")
        _refuse(f"grads[{i}] has {g.numel()} elements, outs[{i}] {o.numel()}", "PM_ERR_SHAPE")

    def pm_clip_gradients(self, max_norm, norm, scale, stream=None):
        """Writes outs, the norm before clipping, and the factor (float32 tensors of one element)."""
        max_norm = float(max_norm)
        if not max_norm > 0:
            _refuse("max_norm must be positive")
        p_norm, p_scale = (_flat(n, t, torch.float32, self.device, t.shape if isinstance(t, torch.Tensor) and t.numel() == 1 else (1,))
                           for n, t in (("norm", norm), ("scale", scale)))
        if p_norm is None or p_scale is None:
            _refuse("norm and scale must be tensors")
        if p_norm == p_scale:
            _refuse("norm and scale share their memory")
        i, j = bisect_left(self.starts, p_norm + 4), bisect_left(self.starts, p_scale + 4)     # the spans that start in front of their ends
        if i and self.stops[i - 1] > p_norm or j and self.stops[j - 1] > p_scale:
            _refuse(f"{'norm' if i and self.stops[i - 1] > p_norm else 'scale'} lies in one of the tensors")
        _launch_with(self.ws_bytes, self.L.pm_clip_gradients, (self.tensors, len(self.tensors), max_norm, p_norm, p_scale), self.device, stream)
