"""Operators on device tensors: a recurrent layer that is parallel over the length, the loss behind it and the update of its parameters.

  decay_attention        o_t = scale * q_t S_t, S_t = lambda_h S_(t-1) + k_t v_t^T over packed sequences
  decay_attention_grad   its gradients with respect to q, k, v and the states that enter
  decay_attention_step   the same recurrence for one new token of each sequence, the states in place
  token_logprobs         log probabilities of labels, entropies and most likely alternatives of rows of scores
  token_logprobs_grad    the gradient of the first two with respect to the scores
  clip_step              the norm of all gradients, and the gradient step (or the gradients) clipped to it

Thin calls over libob.so (include/ob.h holds the full description): tensors of fp32, bf16 or fp16 on the current device, read and
written on torch's current stream; results and scratch memory are torch's.  Nothing waits for the GPU or is copied to or from it, so calls
may be captured into a HIP graph.  Gradients are calls of their own, as the rest of this library has them: autograd records nothing here.  A tensor that
another stream made or will read is ordered by the caller, as for any work on streams.  Arguments that do not fit raise ObError.
"""
from __future__ import annotations

import ctypes
import struct
from array import array
from typing import NamedTuple, Optional

import torch

from .binding import ObError, lib

OB_E_DIM, OB_E_RANGE, OB_E_ARG = -2, -3, -8
OB_TOP_MAX = 64
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_DECAY = struct.Struct("=6iqdQQ" + 7 * "Qqq" + "6Q")
_SCORES = struct.Struct("=6iQqQ8QQq")
_TENSOR = struct.Struct("=QQqii")    # an entry of ob_clip_step's table; written as four 64-bit numbers
_NO_ROWS = (0, 0, 0)


def _call(name, rc):
    if rc < 0:
        raise ObError(rc, (lib().ob_last_error(None) or b"").decode() or name)


def _packed(record, *args):
    try:
        return record.pack(*args)
    except struct.error as e:
        raise ObError(OB_E_RANGE, f"an argument does not fit: {e}")


# torch.cuda.current_stream() builds an object (2.7 us); the address alone takes 0.1, against some 3 us of a launch
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(*tensors):
    """The current stream of the device that the tensors are on, which has to be the current one."""
    at = torch.cuda.current_device() if tensors[0].is_cuda else -2
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ObError(OB_E_ARG, f"tensor on {t.device}: operators work on the current GPU")
    return _raw_stream(at)


def _type(name, t):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ObError(OB_E_ARG, f"{name} is {t.dtype}: fp32, bf16 or fp16 is wanted")
    return code


def _rows(name, t, shape, dtype):
    """(address, token stride, head stride) of [tokens, heads, width]."""
    if t.dtype != dtype:
        raise ObError(OB_E_ARG, f"{name} is {t.dtype}, q is {dtype}")
    if t.shape != shape:
        raise ObError(OB_E_DIM, f"{name} has shape {tuple(t.shape)}: {tuple(shape)} is wanted")
    a, b, c = t.stride()
    if c != 1 and shape[2] > 1:
        raise ObError(OB_E_ARG, f"{name}: the elements of a head have to be neighbours in memory (stride {c})")
    return t.data_ptr(), a, b


def _plane(name, t, shape):
    if t is None:
        return 0
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ObError(OB_E_DIM, f"{name}: a contiguous fp32 tensor of shape {tuple(shape)} is wanted, not {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _widths(q, k, v):
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ObError(OB_E_DIM, "q, k and v have the dimensions tokens, heads, width")
    tokens, heads, dk = q.shape
    kv_heads, dv = v.shape[1:]
    if heads < 1 or kv_heads < 1 or heads % kv_heads:
        raise ObError(OB_E_DIM, f"{heads} heads over {kv_heads} of keys and values")
    if dk < 1 or dv < 1:
        raise ObError(OB_E_DIM, f"widths {dk} and {dv}")
    return tokens, heads, kv_heads, dk, dv


def _decay(log_decay, heads):
    if log_decay.dtype != torch.float32 or log_decay.shape != (heads,) or not log_decay.is_contiguous():
        raise ObError(OB_E_DIM, f"log_decay: a contiguous fp32 tensor of shape ({heads},) is wanted, not {log_decay.dtype} {tuple(log_decay.shape)}")
    return log_decay.data_ptr()


def _offsets(offsets):
    if isinstance(offsets, torch.Tensor):
        if offsets.is_cuda:
            raise ObError(OB_E_ARG, "offsets are host numbers: a list, an array or a CPU tensor")
        offsets = offsets.tolist()
    elif hasattr(offsets, "tolist"):
        offsets = offsets.tolist()
    try:
        a = array("q", offsets)
    except (TypeError, OverflowError):
        raise ObError(OB_E_ARG, "offsets are whole numbers")
    if not a:
        raise ObError(OB_E_RANGE, "offsets hold one number more than there are sequences")
    return a


def _workspace(record, grad):
    need = ctypes.c_uint64()
    _call("ob_decay_workspace", lib().ob_decay_workspace(record, grad, ctypes.byref(need)))
    return torch.empty(need.value, dtype=torch.uint8, device="cuda") if need.value else None


def decay_attention(q, k, v, log_decay, offsets, scale: Optional[float] = None, *, state_in=None, state_out=None):
    """o [tokens, heads, dv] for q [tokens, heads, dk], k [tokens, kv_heads, dk], v [tokens, kv_heads, dv], log_decay [heads] (fp32, <= 0).

    Sequence b has the tokens offsets[b] .. offsets[b + 1] - 1 (host numbers).  state_in, state_out [sequences, heads, dk, dv] (fp32,
    contiguous, apart in memory): the state before the first token (zeros without), and the one behind the last, which is written if given.
    scale: dk ** -0.5 if not given.  Heads may have any strides; the elements of a head are neighbours."""
    s = _stream(q, k, v, log_decay, state_in, state_out)
    tokens, heads, kv_heads, dk, dv = _widths(q, k, v)
    code = _type("q", q)
    off = _offsets(offsets)
    n = len(off) - 1
    shape = (n, heads, dk, dv)
    o = q.new_empty((tokens, heads, dv))
    args = [code, heads, kv_heads, dk, dv, n, tokens, dk ** -0.5 if scale is None else scale, _decay(log_decay, heads), off.buffer_info()[0],
            *_rows("q", q, (tokens, heads, dk), q.dtype), *_rows("k", k, (tokens, kv_heads, dk), q.dtype),
            *_rows("v", v, (tokens, kv_heads, dv), q.dtype), o.data_ptr(), heads * dv, dv, *_NO_ROWS, *_NO_ROWS, *_NO_ROWS,
            _plane("state_in", state_in, shape), _plane("state_out", state_out, shape), 0, 0, 0, 0]
    record = _packed(_DECAY, *args)
    w = _workspace(record, 0)
    if w is not None:
        args[-2:] = w.data_ptr(), w.numel()
        record = _packed(_DECAY, *args)
    _call("ob_decay_attention", lib().ob_decay_attention(s, record))
    return o


def decay_attention_grad(q, k, v, log_decay, offsets, do, scale: Optional[float] = None, *, state_in=None, dstate_out=None, dstate_in=None):
    """(dq, dk, dv) of decay_attention from do, the gradient with respect to o, and dstate_out, that with respect to state_out (zeros without).

    state_in is the one of the forward pass.  dstate_in, if given, is written: the gradient with respect to state_in.  Nothing of the
    forward pass has to be kept but its inputs."""
    s = _stream(q, k, v, log_decay, do, state_in, dstate_out, dstate_in)
    tokens, heads, kv_heads, dk, dv = _widths(q, k, v)
    code = _type("q", q)
    off = _offsets(offsets)
    n = len(off) - 1
    shape = (n, heads, dk, dv)
    dq = q.new_empty((tokens, heads, dk))
    gk = q.new_empty((tokens, kv_heads, dk))
    gv = q.new_empty((tokens, kv_heads, dv))
    args = [code, heads, kv_heads, dk, dv, n, tokens, dk ** -0.5 if scale is None else scale, _decay(log_decay, heads), off.buffer_info()[0],
            *_rows("q", q, (tokens, heads, dk), q.dtype), *_rows("k", k, (tokens, kv_heads, dk), q.dtype),
            *_rows("v", v, (tokens, kv_heads, dv), q.dtype), *_rows("do", do, (tokens, heads, dv), q.dtype),
            dq.data_ptr(), heads * dk, dk, gk.data_ptr(), kv_heads * dk, dk, gv.data_ptr(), kv_heads * dv, dv,
            _plane("state_in", state_in, shape), 0, _plane("dstate_out", dstate_out, shape), _plane("dstate_in", dstate_in, shape), 0, 0]
    record = _packed(_DECAY, *args)
    w = _workspace(record, 1)
    if w is not None:
        args[-2:] = w.data_ptr(), w.numel()
        record = _packed(_DECAY, *args)
    _call("ob_decay_attention_grad", lib().ob_decay_attention_grad(s, record))
    return dq, gk, gv


def decay_attention_step(q, k, v, log_decay, state, scale: Optional[float] = None):
    """o [sequences, heads, dv] of one new token of each sequence; `state` [sequences, heads, dk, dv] (fp32, contiguous) is updated in place."""
    s = _stream(q, k, v, log_decay, state)
    tokens, heads, kv_heads, dk, dv = _widths(q, k, v)
    code, dtype = _type("q", q), q.dtype
    if state is None:
        raise ObError(OB_E_ARG, "no state")
    o = q.new_empty((tokens, heads, dv))
    _call("ob_decay_attention_step", lib().ob_decay_attention_step(s, _packed(
        _DECAY, code, heads, kv_heads, dk, dv, tokens, tokens, dk ** -0.5 if scale is None else scale, _decay(log_decay, heads), 0,
        *_rows("q", q, (tokens, heads, dk), dtype), *_rows("k", k, (tokens, kv_heads, dk), dtype), *_rows("v", v, (tokens, kv_heads, dv), dtype),
        o.data_ptr(), heads * dv, dv, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, _plane("state", state, (tokens, heads, dk, dv)), 0, 0, 0, 0)))
    return o


class TokenLogprobs(NamedTuple):
    """What token_logprobs gives: fp32 [rows], and [rows, top] with int32 classes; row_stats [2, rows] (the largest score of each row, and the sum
    of exp(score - largest)) is for token_logprobs_grad."""
    logprob: torch.Tensor
    entropy: torch.Tensor
    top_logprobs: torch.Tensor
    top_ids: torch.Tensor
    row_stats: torch.Tensor


def _scores(scores, labels):
    if scores.dim() != 2 or labels.dim() != 1 or labels.shape[0] != scores.shape[0]:
        raise ObError(OB_E_DIM, f"scores {tuple(scores.shape)} and labels {tuple(labels.shape)}: [rows, classes] and [rows] are wanted")
    if labels.dtype not in (torch.int32, torch.int64):
        raise ObError(OB_E_ARG, f"labels are {labels.dtype}: int32 or int64 is wanted")
    if labels.shape[0] > 1 and labels.stride(0) != 1:
        raise ObError(OB_E_ARG, "labels have to be neighbours in memory")
    if scores.shape[1] > 1 and scores.stride(1) != 1:
        raise ObError(OB_E_ARG, "the scores of a row have to be neighbours in memory")
    return scores.shape[0], scores.shape[1], 1 if labels.dtype == torch.int64 else 0


def token_logprobs(scores, labels, top: int = 0) -> TokenLogprobs:
    """Log probabilities of labels [rows] (int32 or int64) under softmax of scores [rows, classes], entropies, and the `top` most likely classes.

    A label < 0 is padding (log probability 0); a label >= classes gives NaN.  Scores of -inf are forbidden classes; a row of nothing else
    has log probability -inf and entropy 0.  Alternatives fall; among equal scores the lower class comes first; where none are left: -inf, -1."""
    s = _stream(scores, labels)
    rows, classes, wide = _scores(scores, labels)
    code = _type("scores", scores)
    if not 0 <= top <= min(OB_TOP_MAX, classes):
        raise ObError(OB_E_RANGE, f"{top} alternatives of {classes} classes (at most {OB_TOP_MAX})")
    lp = scores.new_empty(rows, dtype=torch.float32)
    h, stats = lp.new_empty(rows), lp.new_empty((2, rows))
    top_lp, top_id = lp.new_empty((rows, top)), labels.new_empty((rows, top), dtype=torch.int32)
    at = stats.data_ptr()
    _call("ob_token_logprobs", lib().ob_token_logprobs(s, _packed(
        _SCORES, code, wide, rows, classes, top, 0, scores.data_ptr(), scores.stride(0), labels.data_ptr(), lp.data_ptr(), h.data_ptr(), at, at + 4 * rows,
        top_lp.data_ptr(), top_id.data_ptr(), 0, 0, 0, 0)))
    return TokenLogprobs(lp, h, top_lp, top_id, stats)


def token_logprobs_grad(scores, labels, result: TokenLogprobs, dlogprob=None, dentropy=None):
    """The gradient with respect to the scores, in their type, from those with respect to logprob and entropy (fp32 [rows]; zeros without).

    `result` is what token_logprobs gave for the same scores and labels."""
    s = _stream(scores, labels, result.entropy, result.row_stats, dlogprob, dentropy)
    rows, classes, wide = _scores(scores, labels)
    code = _type("scores", scores)
    for name, t, shape in (("entropy", result.entropy, (rows,)), ("row_stats", result.row_stats, (2, rows)), ("dlogprob", dlogprob, (rows,)),
                           ("dentropy", dentropy, (rows,))):
        if t is not None and (t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous()):
            raise ObError(OB_E_DIM, f"{name}: a contiguous fp32 tensor of shape {shape} is wanted, not {t.dtype} {tuple(t.shape)}")
    d = scores.new_empty((rows, classes))
    at = result.row_stats.data_ptr()
    _call("ob_token_logprobs_grad", lib().ob_token_logprobs_grad(s, _packed(
        _SCORES, code, wide, rows, classes, 0, 0, scores.data_ptr(), scores.stride(0), labels.data_ptr(), result.logprob.data_ptr(), result.entropy.data_ptr(),
        at, at + 4 * rows, 0, 0, 0 if dlogprob is None else dlogprob.data_ptr(),
        0 if dentropy is None else dentropy.data_ptr(), d.data_ptr(), classes)))
    return d


def clip_step(grads, max_norm: float, params=None, lr: Optional[float] = None):
    """The norm of all gradients together (fp32, on the device), and with f = min(1, max_norm / norm)

      params -= lr * f * grads   in place, if params (a list of the same shapes) and lr are given,
      grads *= f                 in place without them.

    Tensors are contiguous and may be of different types.  max_norm = math.inf clips nothing."""
    if params is not None and (lr is None or len(params) != len(grads)):
        raise ObError(OB_E_ARG, "parameters come with lr, and one for each gradient")
    n = len(grads)
    s = _stream(grads[0]) if n else _raw_stream(torch.cuda.current_device())
    device = grads[0].get_device() if n else 0
    table = array("q")
    put = table.extend
    for i, g in enumerate(grads):
        p = g if params is None else params[i]
        gt, pt = _TYPES.get(g.dtype), _TYPES.get(p.dtype)
        if gt is None or pt is None:
            raise ObError(OB_E_ARG, f"tensor {i}: fp32, bf16 or fp16 is wanted, not {g.dtype} and {p.dtype}")
        if not (g.is_contiguous() and p.is_contiguous()):
            raise ObError(OB_E_ARG, f"tensor {i} is not contiguous")
        if p.shape != g.shape:
            raise ObError(OB_E_DIM, f"tensor {i}: parameter {tuple(p.shape)}, gradient {tuple(g.shape)}")
        if g.get_device() != device or p.get_device() != device:
            raise ObError(OB_E_ARG, f"tensor {i} is on another device")
        put((g.data_ptr(), 0 if params is None else p.data_ptr(), g.numel(), gt | pt << 32))
    at = table.buffer_info()[0]
    need = ctypes.c_uint64()
    _call("ob_clip_workspace", lib().ob_clip_workspace(at, n, ctypes.byref(need)))
    w = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    norm = torch.empty((), dtype=torch.float32, device="cuda")
    _call("ob_clip_step", lib().ob_clip_step(s, at, n, max_norm, 0.0 if lr is None else lr, norm.data_ptr(), w.data_ptr(), need.value))
    return norm
