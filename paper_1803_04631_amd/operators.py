"""Operators on CUDA tensors for models that are trained and scored next to the sampled topics: layer
norm, log-probabilities of documents' words with entropy and likeliest words, their gradients, and
the global gradient norm with clipping.

Argument marshalling only, like the rest of the binding: everything is computed by the library's
HIP kernels (include/mlda.h says what exactly), on torch's current stream of the tensors' device,
without synchronising it.  Outputs and workspaces come from torch's allocator.  Tensors are fp32, bf16
or fp16; results are sums in fp32 or fp64 that are rounded once.  Nothing is recorded for torch's
differentiation: the backward passes are calls of their own.  An argument that a function does
not take raises ValueError before anything is launched.

Inputs that other streams work on are the caller's to order, as with torch's own operations.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from . import _check, load_library

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # MLDA_FP32, MLDA_BF16, MLDA_FP16
MAX_ALTERNATIVES = 32                                                 # MLDA_MAX_ALTERNATIVES


class TokenLogprobs(NamedTuple):
    logprobs: torch.Tensor                     # [n_tokens] fp32
    stats: torch.Tensor                        # [rows, 2] fp32: greatest logit, ln sum exp(logit - it)
    entropy: Optional[torch.Tensor]            # [rows] fp32
    top_ids: Optional[torch.Tensor]            # [rows, alternatives] int32
    top_logprobs: Optional[torch.Tensor]       # [rows, alternatives] fp32


def _need(ok, message):
    if not ok:
        raise ValueError(message)


def _on(device):
    """The library launches on the current device."""
    _need(device.type == "cuda", "tensors must be on a GPU: there is no CPU path")
    return torch.cuda.device(device)


def _rows(t, name):
    """A matrix's rows, consecutive columns each: (rows, cols, stride)."""
    _need(t.dim() == 2 and t.shape[1] >= 1, f"{name} must be a matrix with at least one column")
    _need(t.dtype in _TYPES, f"{name} must be fp32, bf16 or fp16")
    rows, cols = t.shape
    stride, step = t.stride()
    _need((step == 1 or cols == 1) and (rows <= 1 or stride >= cols),
          f"{name} must have consecutive columns and rows that do not overlap")
    return rows, cols, stride


def _like(t, name, shape, dtype, device):
    """A contiguous tensor of that shape, type and device; its address."""
    _need(tuple(t.shape) == shape and t.dtype == dtype and t.device == device and t.is_contiguous(),
          f"{name} must be a contiguous {dtype} tensor of shape {shape} on {device}")
    return t.data_ptr()


def _out_rows(out, name, like):
    """Rows for a result of the shape and type of `like`."""
    if out is None:
        out = torch.empty(like.shape, dtype=like.dtype, device=like.device)
    else:
        _need(out.shape == like.shape and out.dtype == like.dtype and out.device == like.device,
              f"{name} must have the shape, type and device of the input")
    return out, _rows(out, name)[2]


def _workspace(size_call, args, device):
    n = ctypes.c_size_t()
    _check(size_call(*args, ctypes.addressof(n)))
    if not n.value:
        return None, 0, 0
    t = torch.empty(n.value, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), n.value


def _with_device(fn):
    """Makes the first tensor's device the current one for the call, where it is another."""
    @functools.wraps(fn)
    def call(first, *args, **kwargs):
        device = first.device if isinstance(first, torch.Tensor) else None
        if device is None:
            raise ValueError("a tensor is wanted")
        _need(device.type == "cuda", "tensors must be on a GPU: there is no CPU path")
        if device.index == torch.cuda.current_device():
            return fn(first, *args, **kwargs)
        with torch.cuda.device(device):
            return fn(first, *args, **kwargs)
    return call


def _weight_type(weight, bias, x, cols):
    """The weight's type code and both addresses (0: none)."""
    given = weight if weight is not None else bias
    if given is None:
        return _TYPES[x.dtype], 0, 0
    _need(given.dtype == x.dtype or given.dtype == torch.float32, "weight and bias must have the type of x, or be fp32")
    at = [0 if t is None else _like(t, name, (cols,), given.dtype, x.device) for t, name in ((weight, "weight"), (bias, "bias"))]
    return _TYPES[given.dtype], at[0], at[1]


@_with_device
def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None):
    """Each row of x [rows, cols] less its mean, over its standard deviation, times weight, plus bias.
    Returns (y, mean [rows], rstd [rows]); `out` (x, for instance) takes y."""
    rows, cols, stride = _rows(x, "x")
    kind, at_weight, at_bias = _weight_type(weight, bias, x, cols)
    y, y_stride = _out_rows(out, "out", x)
    mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device).unbind(0)
    _check(load_library().mlda_layer_norm(
        x.data_ptr(), stride, at_weight, at_bias, y.data_ptr(), y_stride, mean.data_ptr(), rstd.data_ptr(), rows, cols,
        eps, _TYPES[x.dtype], kind, torch.cuda.current_stream().cuda_stream))
    return y, mean, rstd


@_with_device
def layer_norm_backward(grad_y, x, mean, rstd, weight=None, out=None):
    """(grad_x, grad_weight, grad_bias) for the gradient grad_y of layer_norm's y; the last two are of
    the weight's type (without a weight: of x's).  `out` (grad_y or x, for instance) takes grad_x."""
    rows, cols, stride = _rows(x, "x")
    _need(grad_y.shape == x.shape and grad_y.dtype == x.dtype and grad_y.device == x.device,
          "grad_y must have the shape, type and device of x")
    grad_stride = _rows(grad_y, "grad_y")[2]
    kind, at_weight, _ = _weight_type(weight, None, x, cols)
    at_mean = _like(mean, "mean", (rows,), torch.float32, x.device)
    at_rstd = _like(rstd, "rstd", (rows,), torch.float32, x.device)
    grad_x, out_stride = _out_rows(out, "out", x)
    grad_weight, grad_bias = torch.empty((2, cols), dtype=x.dtype if weight is None else weight.dtype, device=x.device).unbind(0)
    lib = load_library()
    held, at, size = _workspace(lib.mlda_layer_norm_workspace_bytes, (rows, cols), x.device)
    _check(lib.mlda_layer_norm_backward(
        grad_y.data_ptr(), grad_stride, x.data_ptr(), stride, at_mean, at_rstd, at_weight, grad_x.data_ptr(), out_stride,
        grad_weight.data_ptr(), grad_bias.data_ptr(), rows, cols, _TYPES[x.dtype], kind, at, size,
        torch.cuda.current_stream().cuda_stream))
    return grad_x, grad_weight, grad_bias


def _documents(logits, tokens, row_ptr):
    """Checks logits, tokens and row_ptr; the arguments that the library's calls begin with."""
    rows, vocab, stride = _rows(logits, "logits")
    n = tokens.numel()
    at = _like(tokens, "tokens", (n,), torch.int32, logits.device)
    if row_ptr is None:
        _need(n == rows, "without row_ptr there must be one token to a row")
        at_rows = 0
    else:
        at_rows = _like(row_ptr, "row_ptr", (rows + 1,), torch.int64, logits.device)
    return logits.data_ptr(), stride, rows, vocab, _TYPES[logits.dtype], at, at_rows, n


@_with_device
def token_logprobs(logits, tokens, row_ptr=None, alternatives: int = 0, entropy: bool = False) -> TokenLogprobs:
    """Log-probabilities of tokens (int32 words) under the softmax of their rows of logits [rows, vocab]:
    row r has the tokens row_ptr[r] .. row_ptr[r+1]-1 (int64, on the GPU, its last entry at most the number
    of tokens), or without row_ptr one each.  Tokens below zero are none.  With `alternatives` also each row's
    likeliest words, ties to the lowest; with `entropy` the entropies."""
    args = _documents(logits, tokens, row_ptr)
    rows, vocab, device = args[2], args[3], logits.device
    _need(0 <= alternatives <= min(MAX_ALTERNATIVES, vocab), f"alternatives must be in 0 .. {min(MAX_ALTERNATIVES, vocab)}")
    logprobs = torch.empty(args[7], dtype=torch.float32, device=device)
    stats = torch.empty((rows, 2), dtype=torch.float32, device=device)
    entropies = torch.empty(rows, dtype=torch.float32, device=device) if entropy else None
    top_ids = torch.empty((rows, alternatives), dtype=torch.int32, device=device) if alternatives else None
    top_logprobs = torch.empty((rows, alternatives), dtype=torch.float32, device=device) if alternatives else None
    lib = load_library()
    held, at, size = _workspace(lib.mlda_token_logprobs_workspace_bytes, (rows, vocab, alternatives, args[4]), device)
    _check(lib.mlda_token_logprobs(
        *args, alternatives, logprobs.data_ptr(), stats.data_ptr(), entropies.data_ptr() if entropy else 0,
        top_ids.data_ptr() if alternatives else 0, top_logprobs.data_ptr() if alternatives else 0, at, size,
        torch.cuda.current_stream().cuda_stream))
    return TokenLogprobs(logprobs, stats, entropies, top_ids, top_logprobs)


@_with_device
def token_logprobs_backward(grad_logprobs, logits, tokens, stats, row_ptr=None, grad_entropy=None, entropy=None, out=None):
    """The gradient with respect to the logits, for gradients grad_logprobs [n_tokens] of token_logprobs'
    log-probabilities and grad_entropy [rows] (with `entropy` as it came out) of its entropies.  `out` (logits, for
    instance) takes it."""
    args = _documents(logits, tokens, row_ptr)
    rows, device = args[2], logits.device
    at_grad = _like(grad_logprobs, "grad_logprobs", (args[7],), torch.float32, device)
    at_stats = _like(stats, "stats", (rows, 2), torch.float32, device)
    at_entropy = at_grad_entropy = 0
    if grad_entropy is not None:
        _need(entropy is not None, "a gradient of the entropy needs the entropy")
        at_grad_entropy = _like(grad_entropy, "grad_entropy", (rows,), torch.float32, device)
        at_entropy = _like(entropy, "entropy", (rows,), torch.float32, device)
    grad_logits, out_stride = _out_rows(out, "out", logits)
    _check(load_library().mlda_token_logprobs_backward(
        *args, at_stats, at_grad, at_entropy, at_grad_entropy, grad_logits.data_ptr(), out_stride,
        torch.cuda.current_stream().cuda_stream))
    return grad_logits


@_with_device
def token_logprobs_grad(logits, tokens, weights, row_ptr=None, out=None):
    """A training step's loss and gradient in one: (log-probabilities of the tokens, the gradient of
    sum(weights * log-probabilities) with respect to the logits), weights [n_tokens] fp32.  `out` (logits, for
    instance) takes the gradient."""
    args = _documents(logits, tokens, row_ptr)
    device = logits.device
    at_weights = _like(weights, "weights", (args[7],), torch.float32, device)
    logprobs = torch.empty(args[7], dtype=torch.float32, device=device)
    grad_logits, out_stride = _out_rows(out, "out", logits)
    lib = load_library()
    held, at, size = _workspace(lib.mlda_token_logprobs_workspace_bytes, (args[2], args[3], 0, args[4]), device)
    _check(lib.mlda_token_logprobs_grad(
        *args, at_weights, logprobs.data_ptr(), grad_logits.data_ptr(), out_stride, at, size,
        torch.cuda.current_stream().cuda_stream))
    return logprobs, grad_logits


def _tensor_list(tensors, name, device):
    """Addresses, sizes and type codes of contiguous tensors on the device, as host arrays."""
    n = len(tensors)
    for t in tensors:
        _need(t.is_contiguous() and t.device == device and t.dtype in _TYPES,
              f"{name} must be contiguous fp32, bf16 or fp16 tensors on one GPU")
    return ((ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors]), (ctypes.c_int64 * n)(*[t.numel() for t in tensors]),
            (ctypes.c_int32 * n)(*[_TYPES[t.dtype] for t in tensors]))


def _grads(tensors, max_norm, out):
    tensors = list(tensors)
    _need(len(tensors) > 0, "there must be at least one tensor")
    device = tensors[0].device
    with _on(device):
        at, sizes, types = _tensor_list(tensors, "tensors", device)
        norm = torch.empty((), dtype=torch.float32, device=device)
        lib = load_library()
        held, workspace, size = _workspace(lib.mlda_grad_norm_workspace_bytes, (len(tensors),), device)
        stream = torch.cuda.current_stream().cuda_stream
        if max_norm is None:
            _check(lib.mlda_grad_norm(at, sizes, types, len(tensors), norm.data_ptr(), workspace, size, stream))
            return norm
        to = at
        if out is not None:
            out = list(out)
            _need(len(out) == len(tensors) and all(o.dtype == t.dtype and o.shape == t.shape for o, t in zip(out, tensors)),
                  "out must have a tensor of the shape and type of each of tensors")
            to = _tensor_list(out, "out", device)[0]
        _check(lib.mlda_clip_grads(at, to, sizes, types, len(tensors), max_norm, norm.data_ptr(), workspace, size, stream))
        return norm


def grad_norm(tensors):
    """The norm over all tensors of a gradient: the square root of the sum of all squares, as a scalar
    tensor."""
    return _grads(tensors, None, None)


def clip_grads(tensors, max_norm: float, out=None):
    """Scales the tensors of a gradient, in place or into those of `out`, by max_norm / norm where their norm
    exceeds max_norm; a norm that is not finite scales nothing.  Returns the norm before."""
    return _grads(tensors, max_norm, out)
