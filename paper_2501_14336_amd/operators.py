"""Operators on rows of logits beside the selection, on torch tensors: ``logprobs``, ``distill`` and ``route``.

What a language model's rows are used for once they are there: the log probabilities of given tokens with the row's
entropy and its best alternatives (serving, scoring, policy gradients), the divergence from a teacher's top logits (the
lists that ``binding.topk`` keeps of a teacher's rows), and the choice of experts for each token.  Each has its gradient:
``logprobs_backward``, ``distill_backward`` and ``route_backward`` are the calls, and the three operators go through
``torch.autograd`` where their logits ask for a gradient.

Everything runs in the HIP kernels of the C-ABI library (include/rtopk.h holds the formulas and the limits); these functions check
arguments, supply memory and the current stream, and raise ``RtopkError`` for what the kernels do not take.  Nothing
synchronises.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as _B
from .binding import RTOPK_BF16, RTOPK_F16, RTOPK_F32, RtopkError

ROUTE_SIGMOID, ROUTE_RENORMALIZE, ROUTE_GROUP_TOP2 = 1, 2, 4
DISTILL_ROW_STATS = 8

_CODES = {torch.float32: RTOPK_F32, torch.float16: RTOPK_F16, torch.bfloat16: RTOPK_BF16}


class LogProbs(NamedTuple):
    logprobs: torch.Tensor                   # [batch, m] float32
    top_logprobs: Optional[torch.Tensor]     # [batch, k] float32, None for k = 0
    top_indices: Optional[torch.Tensor]      # [batch, k] int64, None for k = 0
    entropy: Optional[torch.Tensor]          # [batch] float32, None unless asked for
    row_stats: torch.Tensor                  # [batch, 2] float32: maximum M and S = sum exp((x - M) / T)


def _refuse(message):
    raise RtopkError(1, message)


def _check(status):
    if status != _B.RTOPK_OK:
        raise RtopkError(status, _B.rtopk_status_string(status))


def _rows(x, what):
    """(address, batch, n, row stride, type) of a [batch, n] tensor whose rows are contiguous."""
    shape = x.shape
    if not x.is_cuda:
        _refuse("%s must live on the GPU; there is no CPU path" % what)
    if len(shape) != 2:
        _refuse("%s must be a [batch, n] tensor" % what)
    batch, n = shape
    if batch < 1 or n < 1:
        _refuse("%s is empty" % what)
    stride = n
    if not x.is_contiguous():
        if batch > 1:
            stride = x.stride(0)
        if (n > 1 and x.stride(1) != 1) or stride < n:
            _refuse("%s must have contiguous rows that do not overlap" % what)
    code = _CODES.get(x.dtype)
    if code is None:
        _refuse("%s must be float32, float16 or bfloat16" % what)
    return x.data_ptr(), batch, n, stride, code


def _address(t, x, shape, dtype, what):
    """The address of a contiguous tensor beside the logits ``x``; None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != x.get_device() or not t.is_contiguous():
        _refuse("%s must be a contiguous %s tensor of shape %s on %s" % (what, dtype, tuple(shape), x.device))
    return t.data_ptr()


def _inverse(temperature):
    temperature = float(temperature)
    if not temperature > 0.0:
        _refuse("temperature must be positive")
    return 1.0 / temperature


# (a stream's handle without the object around it: 0.1 us instead of 2, where a call's own work takes 5)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _enqueue(x, call, *args):
    """The C call with the stream that is current on x's device, which is made current if it is not."""
    device = x.get_device()
    if device == torch.cuda.current_device():
        status = call(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            status = call(*args, _raw_stream(device))
    if status != _B.RTOPK_OK:
        raise RtopkError(status, _B.rtopk_status_string(status))


def _tokens_2d(tokens):
    return tokens if tokens is None or tokens.dim() == 2 else tokens[:, None]


def _workspace(workspace, need, x):
    if workspace is None or workspace.numel() * workspace.element_size() < need or workspace.device != x.device:
        return torch.empty(need, dtype=torch.uint8, device=x.device)
    return workspace


def _gradient(out, x, what="out"):
    if out is None:
        return torch.empty_like(x, memory_format=torch.contiguous_format)
    if out.shape != x.shape or out.dtype is not x.dtype or out.device != x.device:
        _refuse("%s must be like the logits" % what)
    return out


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------

_sizes = {}


def _size(lib, name, *args):
    """A workspace's size; sizes depend on the arguments alone, and are remembered."""
    key = (name,) + args
    need = _sizes.get(key)
    if need is None:
        out = _B.ctypes.c_size_t(0)
        _check(getattr(lib, name)(*args, _B.ctypes.byref(out)))
        if len(_sizes) > 4096:
            _sizes.clear()
        need = _sizes[key] = int(out.value)
    return need


def _logprobs(logits, tokens, k, inv_temperature, entropy, workspace):
    lib = _B.load()
    x, batch, n, stride, code = _rows(logits, "logits")
    m = 0 if tokens is None else tokens.shape[1]
    t = None if tokens is None else _address(tokens, logits, (batch, m), torch.int64, "tokens")
    if not 0 <= k <= n:
        _refuse("k must lie between 0 and the row's length")
    new = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
    lp, stats = new((batch, m)), new((batch, 2))
    h = new((batch,)) if entropy else None
    top, at = (new((batch, k)), new((batch, k), torch.int64)) if k else (None, None)
    need = _size(lib, "rtopk_logprobs_workspace_bytes", batch, n, m, k, code)
    ws = _workspace(workspace, need, logits)
    _enqueue(logits, lib.rtopk_logprobs, x, batch, n, stride, code, inv_temperature, t, m, k, lp.data_ptr(), h.data_ptr() if entropy else None,
             stats.data_ptr(), top.data_ptr() if k else None, at.data_ptr() if k else None, ws.data_ptr(), ws.numel() * ws.element_size())
    return LogProbs(lp, top, at, h, stats)


class _LogProbsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, k, temperature, entropy, workspace):
        r = _logprobs(logits.detach(), tokens, k, _inverse(temperature), entropy, workspace)
        ctx.temperature = temperature
        ctx.save_for_backward(logits, tokens, r.row_stats, r.entropy)
        ctx.mark_non_differentiable(*[t for t in (r.top_logprobs, r.top_indices, r.row_stats) if t is not None])
        return tuple(r)

    @staticmethod
    def backward(ctx, g_logprobs, g_top, g_at, g_entropy, g_stats):
        logits, tokens, row_stats, entropy = ctx.saved_tensors
        grad = logprobs_backward(logits.detach(), tokens, row_stats, None if tokens is None else g_logprobs.contiguous(), entropy,
                                 None if entropy is None else g_entropy.contiguous(), ctx.temperature)
        return grad, None, None, None, None, None


def logprobs(logits, tokens=None, k: int = 0, temperature: float = 1.0, entropy: bool = False, workspace=None) -> LogProbs:
    """Log probabilities under softmax(logits / temperature), row by row.

    ``logits`` [batch, n]: float32, float16 or bfloat16, rows contiguous.  ``tokens`` [batch] or [batch, m] int64: whose log probability
    is wanted; a negative token is padding (0, no gradient).  ``k``: how many alternatives, best first, lowest index first among equals.
    ``entropy``: whether to return it.  ``workspace``: a uint8 tensor to use again from call to call.

    Differentiable in ``logprobs`` and ``entropy``, not in the alternatives (give their indices as tokens for that).
    """
    tokens = _tokens_2d(tokens)
    if torch.is_grad_enabled() and logits.requires_grad:
        return LogProbs(*_LogProbsFunction.apply(logits, tokens, k, temperature, entropy, workspace))
    return _logprobs(logits, tokens, k, _inverse(temperature), entropy, workspace)


def logprobs_backward(logits, tokens, row_stats, grad_logprobs, entropy=None, grad_entropy=None, temperature: float = 1.0, out=None):
    """The gradient to the logits of sum(grad_logprobs * logprobs) + sum(grad_entropy * entropy); ``row_stats`` and ``entropy`` are what
    ``logprobs`` returned for the same logits and temperature.  ``out``: a tensor like the logits to write into."""
    lib = _B.load()
    tokens = _tokens_2d(tokens)
    x, batch, n, stride, code = _rows(logits, "logits")
    m = 0 if tokens is None else tokens.shape[1]
    if m and grad_logprobs is None:
        _refuse("grad_logprobs is missing")
    if grad_entropy is not None and entropy is None:
        _refuse("grad_entropy needs the entropy")
    if m and grad_logprobs.dim() == 1:
        grad_logprobs = grad_logprobs[:, None]
    out = _gradient(out, logits)
    g, g_batch, g_n, g_stride, _ = _rows(out, "out")
    f32 = torch.float32
    args = (_address(tokens, logits, (batch, m), torch.int64, "tokens") if m else None, m,
            _address(row_stats, logits, (batch, 2), f32, "row_stats"),
            _address(grad_logprobs, logits, (batch, m), f32, "grad_logprobs") if m else None,
            _address(entropy, logits, (batch,), f32, "entropy"), _address(grad_entropy, logits, (batch,), f32, "grad_entropy"))
    _enqueue(logits, lib.rtopk_logprobs_backward, x, batch, n, stride, code, _inverse(temperature), *args, g, g_stride)
    return out


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def _lists(student, values, indices, teacher_lse, temperature):
    """The arguments that the distillation calls have in common."""
    x, batch, n, stride, code = _rows(student, "student")
    if indices.dim() != 2 or indices.shape[1] < 1:
        _refuse("teacher_indices must be a [batch, k] tensor")
    k = indices.shape[1]
    value_code = _CODES.get(values.dtype)
    if value_code is None:
        _refuse("teacher_values must be float32, float16 or bfloat16")
    return (x, batch, n, stride, code, _inverse(temperature), _address(values, student, (batch, k), values.dtype, "teacher_values"), value_code,
            _address(indices, student, (batch, k), torch.int64, "teacher_indices"), k,
            _address(teacher_lse, student, (batch,), torch.float32, "teacher_lse"))


def _distill(student, values, indices, teacher_lse, temperature, workspace):
    lib = _B.load()
    args = _lists(student, values, indices, teacher_lse, temperature)
    batch, n, code, k = args[1], args[2], args[4], args[9]
    loss = torch.empty((batch,), dtype=torch.float32, device=student.device)
    stats = torch.empty((batch, DISTILL_ROW_STATS), dtype=torch.float32, device=student.device)
    ws = _workspace(workspace, _size(lib, "rtopk_distill_workspace_bytes", batch, n, k, code), student)
    _enqueue(student, lib.rtopk_distill, *args, loss.data_ptr(), stats.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size())
    return loss, stats


class _DistillFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, student, values, indices, teacher_lse, temperature, workspace):
        loss, stats = _distill(student.detach(), values, indices, teacher_lse, temperature, workspace)
        ctx.temperature = temperature
        ctx.save_for_backward(student, values, indices, stats, teacher_lse)
        ctx.mark_non_differentiable(stats)
        return loss, stats

    @staticmethod
    def backward(ctx, g_loss, g_stats):
        student, values, indices, stats, teacher_lse = ctx.saved_tensors
        grad = distill_backward(student.detach(), values, indices, stats, g_loss.contiguous(), teacher_lse, ctx.temperature)
        return grad, None, None, None, None, None


def distill(student, teacher_values, teacher_indices, teacher_lse=None, temperature: float = 1.0, workspace=None):
    """Per row, the divergence of softmax(student / temperature) from a teacher's top logits: (loss [batch], row_stats [batch, 8]), float32.

    ``student`` [batch, n]; ``teacher_values`` [batch, k], any of the three types, and ``teacher_indices`` [batch, k] int64 are what
    ``binding.topk`` keeps of the teacher's rows, distinct within a row; a negative index is padding.  Without ``teacher_lse`` the teacher's
    distribution is the softmax over its list.  ``teacher_lse`` [batch]: the teacher's log-sum over its whole row at this temperature
    (``logprobs``' row_stats give it); what is not listed is then one class more.  The loss is not multiplied by temperature ** 2.

    Differentiable in ``student``.
    """
    if torch.is_grad_enabled() and student.requires_grad:
        return _DistillFunction.apply(student, teacher_values, teacher_indices, teacher_lse, temperature, workspace)
    return _distill(student, teacher_values, teacher_indices, teacher_lse, temperature, workspace)


def distill_backward(student, teacher_values, teacher_indices, row_stats, grad_loss, teacher_lse=None, temperature: float = 1.0, out=None):
    """The gradient of sum(grad_loss * loss) to the student's logits; ``row_stats`` is what ``distill`` returned for the same arguments.
    Rows whose grad_loss is 0 get zeros, whatever they hold.  ``out``: a tensor like the logits to write into."""
    lib = _B.load()
    args = _lists(student, teacher_values, teacher_indices, teacher_lse, temperature)
    out = _gradient(out, student)
    g, _, _, g_stride, _ = _rows(out, "out")
    stats = _address(row_stats, student, (args[1], DISTILL_ROW_STATS), torch.float32, "row_stats")
    w = _address(grad_loss, student, (args[1],), torch.float32, "grad_loss")
    _enqueue(student, lib.rtopk_distill_backward, *args, stats, w, g, g_stride)
    return out


def distill_step(student, teacher_values, teacher_indices, row_weights, teacher_lse=None, temperature: float = 1.0, workspace=None, out=None):
    """``distill`` and its gradient in one call, for loops that know the rows' weights beforehand: (loss [batch], gradient of
    sum(row_weights * loss) to the student).  ``out``: a tensor like the logits for the gradient."""
    lib = _B.load()
    args = _lists(student, teacher_values, teacher_indices, teacher_lse, temperature)
    batch, n, code, k = args[1], args[2], args[4], args[9]
    loss = torch.empty((batch,), dtype=torch.float32, device=student.device)
    out = _gradient(out, student)
    g, _, _, g_stride, _ = _rows(out, "out")
    w = _address(row_weights, student, (batch,), torch.float32, "row_weights")
    ws = _workspace(workspace, _size(lib, "rtopk_distill_workspace_bytes", batch, n, k, code), student)
    _enqueue(student, lib.rtopk_distill_step, *args, w, loss.data_ptr(), g, g_stride, ws.data_ptr(), ws.numel() * ws.element_size())
    return loss, out


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------

def _route_flags(score, renormalize, group_score="max"):
    if score not in ("softmax", "sigmoid") or group_score not in ("max", "top2"):
        _refuse("score is softmax or sigmoid, group_score max or top2")
    return (ROUTE_SIGMOID if score == "sigmoid" else 0) | (ROUTE_RENORMALIZE if renormalize else 0) | (ROUTE_GROUP_TOP2 if group_score == "top2" else 0)


def _route(logits, k, flags, bias, groups, topk_groups, scale, counts):
    lib = _B.load()
    x, tokens, experts, stride, code = _rows(logits, "logits")
    weights = torch.empty((tokens, max(k, 0)), dtype=torch.float32, device=logits.device)
    chosen = torch.empty((tokens, max(k, 0)), dtype=torch.int64, device=logits.device)
    b = _address(bias, logits, (experts,), torch.float32, "bias")
    c = _address(counts, logits, (experts,), torch.int64, "counts")
    _enqueue(logits, lib.rtopk_route, x, tokens, experts, stride, code, b, groups, topk_groups, k, flags, scale, weights.data_ptr(),
             chosen.data_ptr(), c)
    return weights, chosen


class _RouteFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, flags, bias, groups, topk_groups, scale, counts):
        weights, chosen = _route(logits.detach(), k, flags, bias, groups, topk_groups, scale, counts)
        ctx.flags, ctx.scale = flags, scale
        ctx.save_for_backward(logits, chosen)
        ctx.mark_non_differentiable(chosen)
        return weights, chosen

    @staticmethod
    def backward(ctx, g_weights, g_chosen):
        logits, chosen = ctx.saved_tensors
        return (_route_backward(logits.detach(), chosen, g_weights.contiguous(), ctx.flags, ctx.scale, None),) + (None,) * 7


def route(logits, k: int, score: str = "softmax", bias=None, groups: int = 1, topk_groups: int = 1, group_score: str = "max",
          renormalize: bool = True, scale: float = 1.0, counts=None):
    """The k best experts of each token and their weights: (weights [tokens, k] float32, experts [tokens, k] int64), best first.

    ``logits`` [tokens, experts].  ``score``: "softmax" or "sigmoid" of the logits.  ``bias`` [experts] float32 is added to the scores for the choice
    alone.  With ``groups`` > 1 the experts are in that many groups of neighbours, and only the ``topk_groups`` groups with the highest best
    score ("max") or sum of their two best ("top2") are chosen from.  ``renormalize``: weights are divided by their sum.  All are multiplied by
    ``scale``.  ``counts`` [experts] int64: each expert's tokens are added to it.

    Differentiable in the weights; neither the choice nor the bias has a gradient.
    """
    flags = _route_flags(score, renormalize, group_score)
    if torch.is_grad_enabled() and logits.requires_grad:
        return _RouteFunction.apply(logits, k, flags, bias, groups, topk_groups, scale, counts)
    return _route(logits, k, flags, bias, groups, topk_groups, scale, counts)


def _route_backward(logits, experts, grad_weights, flags, scale, out):
    lib = _B.load()
    x, tokens, n, stride, code = _rows(logits, "logits")
    if experts.dim() != 2:
        _refuse("experts must be a [tokens, k] tensor")
    k = experts.shape[1]
    out = _gradient(out, logits)
    g, _, _, g_stride, _ = _rows(out, "out")
    e = _address(experts, logits, (tokens, k), torch.int64, "experts")
    w = _address(grad_weights, logits, (tokens, k), torch.float32, "grad_weights")
    _enqueue(logits, lib.rtopk_route_backward, x, tokens, n, stride, code, e, k, flags, scale, w, g, g_stride)
    return out


def route_backward(logits, experts, grad_weights, score: str = "softmax", renormalize: bool = True, scale: float = 1.0, out=None):
    """The weights' gradient to the logits; ``experts`` is what ``route`` returned for them, the rest its arguments."""
    return _route_backward(logits, experts, grad_weights, _route_flags(score, renormalize), scale, out)
