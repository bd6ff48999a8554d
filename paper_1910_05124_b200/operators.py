"""Operators for programs with their own forward and backward pass, next to `FlatUpdate`: attention over packed sequences,
log probabilities of given tokens, and gradient clipping.  Argument checks and marshalling only; the tensors belong to the
caller, outputs included.

Every call is asynchronous on `stream` (default: the current stream of the tensors' device) and may be captured into a CUDA
graph.  As with any CUDA call, a tensor that another stream still writes has to be waited for by the caller, and a tensor
that belongs to another stream has to be kept until the call has run.  Refused arguments raise PipeMareError.
"""
import ctypes as C
from bisect import bisect_left

import torch

from .binding import (PM_BF16, PM_F32, PipeMareError, _check, lib, pm_attention_desc, pm_head_view, pm_tensor_pair)

_DTYPES = {torch.float32: PM_F32, torch.bfloat16: PM_BF16}
_VIEW = C.sizeof(pm_head_view)


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
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device.index and t.shape == shape and t.is_contiguous()):
        _mismatch(name, t, dtype, device, shape)
    return t.data_ptr()


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


def _launch(call, device, stream, workspace=0):
    """call(stream handle[, workspace pointer]) with the tensors' device current, and its status checked.

    The workspace is device scratch of this call alone: it comes from the allocator's pool of the launching stream, so the
    memory is reused only by work queued behind the call (under capture it stays with the graph)."""
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _launch(call, device, stream, workspace)
    if stream is None:
        handle = _raw_stream(device.index)
    else:
        if stream.device != device:
            _refuse(f"the stream belongs to {stream.device}, the tensors to {device}")
        handle = stream.cuda_stream
    if not workspace:
        return _check(call(handle))
    if stream is None or handle == _raw_stream(device.index):
        scratch = torch.empty(workspace, dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(stream):
            scratch = torch.empty(workspace, dtype=torch.uint8, device=device)
    return _check(call(handle, scratch.data_ptr()))


class PackedAttention:
    """Attention over sequences of different lengths laid end to end, with shared key/value heads.

    q, o: [tokens, n_heads, head_dim]; k, v: [tokens, n_kv_heads, head_dim]; all float32 or all bfloat16, the last dimension
    contiguous, the others at any stride (q, k and v may be views of one projection's output).  cu_seqlens: int32
    [sequences + 1] on the device, ascending; sequence b is tokens cu_seqlens[b] to cu_seqlens[b + 1] - 1, and tokens outside
    all sequences are neither used nor written.  lse: float32 [n_heads, tokens].  head_dim up to 128.
    """

    def __init__(self, n_heads, n_kv_heads, head_dim, *, causal=True, scale=None):
        if n_heads < 1 or n_kv_heads < 1 or n_heads % n_kv_heads:
            _refuse("n_heads must be a positive multiple of n_kv_heads")
        if head_dim < 1:
            _refuse("head_dim must be positive")
        if head_dim > 128:
            _refuse("heads wider than 128", "PM_ERR_UNSUPPORTED")
        scale = head_dim ** -0.5 if scale is None else float(scale)
        if not 0 < scale < 2e38:
            _refuse("scale must be positive and below 2e38")
        self.n_heads, self.n_kv_heads, self.head_dim, self.causal, self.scale = n_heads, n_kv_heads, head_dim, bool(causal), scale
        self.L = lib()

    def _desc(self, q, cu_seqlens):
        device = _compute_device("q", q)
        if q.dim() != 3:
            _refuse(f"q has shape {tuple(q.shape)}, expected [tokens, {self.n_heads}, {self.head_dim}]", "PM_ERR_SHAPE")
        if not isinstance(cu_seqlens, torch.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
            _refuse("cu_seqlens must be a one-dimensional tensor of sequences + 1 entries", "PM_ERR_SHAPE")
        cu = _flat("cu_seqlens", cu_seqlens, torch.int32, device, cu_seqlens.shape)
        tokens = q.shape[0]
        return device, tokens, C.byref(pm_attention_desc(_DTYPES[q.dtype], self.n_heads, self.n_kv_heads, self.head_dim,
                                                         cu_seqlens.numel() - 1, self.causal, tokens, self.scale)), cu

    def _views(self, tokens, dtype, device, names, tensors, heads, n_read):
        """One array of pm_head_view for tensors with `heads` heads each, checked; those behind the first n_read are written."""
        d, index, flat = self.head_dim, device.index, []
        for t, h in zip(tensors, heads):
            if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == index and t.shape == (tokens, h, d)):
                _mismatch(names[len(flat) // 3], t, dtype, device, (tokens, h, d))
            token, head, one = t.stride()
            if one != 1 and d > 1:
                _refuse(f"the last dimension of {names[len(flat) // 3]} must be contiguous")
            if (head != d or token < h * d) and len(flat) >= 3 * n_read:
                self._check_apart(names[len(flat) // 3], ((token, tokens), (head, h)))
            flat += (t.data_ptr(), token, head)
        return (C.c_int64 * len(flat))(*flat)

    def _check_apart(self, name, dims):
        """Rows of one head, or heads of one row, of a tensor that is written must not share elements."""
        if min(n for _, n in dims) < 1:
            return
        end = self.head_dim
        for stride, n in sorted((s, n) for s, n in dims if n > 1):
            if stride < end:
                _refuse(f"{name} overlaps itself")
            end += stride * (n - 1)

    def pm_attention_packed_forward(self, q, k, v, cu_seqlens, o, lse=None, stream=None):
        """Writes o and, for a backward pass, lse."""
        device, tokens, desc, cu = self._desc(q, cu_seqlens)
        H, K = self.n_heads, self.n_kv_heads
        views = self._views(tokens, q.dtype, device, ("q", "k", "v", "o"), (q, k, v, o), (H, K, K, H), 3)
        p_lse = _flat("lse", lse, torch.float32, device, (H, tokens))
        at = C.addressof(views)
        _launch(lambda st: self.L.pm_attention_packed_forward(desc, at, at + _VIEW, at + 2 * _VIEW, cu, at + 3 * _VIEW, p_lse, st), device, stream)

    def pm_attention_packed_backward(self, q, k, v, o, lse, d_o, cu_seqlens, dq, dk, dv, stream=None):
        """Writes dq, dk and dv from d_o and what the forward call wrote."""
        device, tokens, desc, cu = self._desc(q, cu_seqlens)
        if lse is None:
            _refuse("lse must be a tensor")
        H, K = self.n_heads, self.n_kv_heads
        views = self._views(tokens, q.dtype, device, ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"), (q, k, v, o, d_o, dq, dk, dv),
                            (H, K, K, H, H, H, K, K), 5)
        p_lse = _flat("lse", lse, torch.float32, device, (H, tokens))
        at = C.addressof(views)
        need = self.L.pm_attention_packed_workspace_bytes(desc)
        _launch(lambda st, ws=None: self.L.pm_attention_packed_backward(
            desc, at, at + _VIEW, at + 2 * _VIEW, at + 3 * _VIEW, p_lse, at + 4 * _VIEW, cu, at + 5 * _VIEW, at + 6 * _VIEW, at + 7 * _VIEW, ws, need, st),
            device, stream, need)

    def pm_attention_packed_status(self, device="cuda", stream=None):
        """Raises if a device-side wait of a tensor-core kernel ran out since the last call on this device (a defect); synchronises
        the stream."""
        _launch(self.L.pm_attention_packed_status, _indexed(device), stream)

    def pm_attention_packed_selftest_wait_timeout(self, limit_cycles, device="cuda", stream=None):
        """Enqueues a wait that runs out after limit_cycles: the next pm_attention_packed_status on this device raises."""
        _launch(lambda st: self.L.pm_attention_packed_selftest_wait_timeout(int(limit_cycles), st), _indexed(device), stream)


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
        _launch(lambda st: self.L.pm_token_logprobs(*args, st), device, stream)

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
        _launch(lambda st: self.L.pm_token_logprobs_backward(*args, st), device, stream)


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
        _launch(lambda st, ws: self.L.pm_clip_gradients(self.tensors, len(self.tensors), max_norm, p_norm, p_scale, ws, self.ws_bytes, st),
                self.device, stream, self.ws_bytes)
