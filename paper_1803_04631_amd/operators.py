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


# On one document a call takes the GPU 4 us; what is done here for it is kept short: messages are made where one is
# raised, sizes of workspaces are asked for once.
def _launch(device, call, *args):
    """The library's call on the current stream of that device, which it wants to be the current one."""
    index = device.index
    if index == torch.cuda.current_device():
        rc = call(*args, torch._C._cuda_getCurrentRawStream(index))    # current_stream().cuda_stream, which takes 2.7 us
    else:
        with torch.cuda.device(device):
            rc = call(*args, torch._C._cuda_getCurrentRawStream(index))
    if rc:
        _check(rc)


def _rows(t, name):
    """A matrix's rows, consecutive columns each: (rows, cols, stride, type code)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU: there is no CPU path")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{name} must be fp32, bf16 or fp16")
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{name} must be a matrix with at least one column")
    rows, cols = t.shape
    stride, step = t.stride()
    if (step != 1 and cols != 1) or (rows > 1 and stride < cols):
        raise ValueError(f"{name} must have consecutive columns and rows that do not overlap")
    return rows, cols, stride, kind


def _like(t, name, shape, dtype, device):
    """The address of a contiguous tensor of that shape, type and device."""
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _rows_like(t, name, like):
    """The stride of rows of the shape, type and device of `like`."""
    stride = _rows(t, name)[2]
    if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name} must have the shape, type and device of the input")
    return stride


def _fp32(shape, device):
    return torch.empty(shape, dtype=torch.float32, device=device)


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(call, *sizes):
    n = ctypes.c_size_t()
    _check(getattr(load_library(), call)(*sizes, ctypes.addressof(n)))
    return n.value


def _workspace(size, device):
    """(what holds the memory, its address)"""
    if not size:
        return None, 0
    t = torch.empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _columns(t, name, cols, x):
    """The address of a weight or bias, and its type code."""
    if not isinstance(t, torch.Tensor) or (t.dtype != x.dtype and t.dtype != torch.float32):
        raise ValueError(f"{name} must have the type of x, or be fp32")
    return _like(t, name, (cols,), t.dtype, x.device), _TYPES[t.dtype]


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None):
    """Each row of x [rows, cols] less its mean, over its standard deviation, times weight, plus bias.
    Returns (y, mean [rows], rstd [rows]); `out` (x, for instance) takes y."""
    rows, cols, stride, kind = _rows(x, "x")
    device = x.device
    at_weight = at_bias = 0
    weight_kind = kind
    if weight is not None:
        at_weight, weight_kind = _columns(weight, "weight", cols, x)
    if bias is not None:
        at_bias, bias_kind = _columns(bias, "bias", cols, x)
        if weight is not None and bias_kind != weight_kind:
            raise ValueError("bias must have the type of weight")
        weight_kind = bias_kind
    if out is None:
        out = torch.empty_like(x)
    out_stride = _rows_like(out, "out", x)
    mean, rstd = _fp32(rows, device), _fp32(rows, device)
    _launch(device, load_library().mlda_layer_norm, x.data_ptr(), stride, at_weight, at_bias, out.data_ptr(), out_stride,
            mean.data_ptr(), rstd.data_ptr(), rows, cols, eps, kind, weight_kind)
    return out, mean, rstd


def layer_norm_backward(grad_y, x, mean, rstd, weight=None, out=None):
    """(grad_x, grad_weight, grad_bias) for the gradient grad_y of layer_norm's y; the last two are of
    the weight's type (without a weight: of x's).  `out` (grad_y or x, for instance) takes grad_x."""
    rows, cols, stride, kind = _rows(x, "x")
    device = x.device
    grad_stride = _rows_like(grad_y, "grad_y", x)
    at_weight, weight_kind, dtype = 0, kind, x.dtype
    if weight is not None:
        at_weight, weight_kind = _columns(weight, "weight", cols, x)
        dtype = weight.dtype
    at_mean = _like(mean, "mean", (rows,), torch.float32, device)
    at_rstd = _like(rstd, "rstd", (rows,), torch.float32, device)
    if out is None:
        out = torch.empty_like(x)
    out_stride = _rows_like(out, "out", x)
    grad_weight = torch.empty(cols, dtype=dtype, device=device)
    grad_bias = torch.empty(cols, dtype=dtype, device=device)
    size = _workspace_bytes("mlda_layer_norm_workspace_bytes", rows, cols)
    held, at = _workspace(size, device)
    _launch(device, load_library().mlda_layer_norm_backward, grad_y.data_ptr(), grad_stride, x.data_ptr(), stride, at_mean, at_rstd,
            at_weight, out.data_ptr(), out_stride, grad_weight.data_ptr(), grad_bias.data_ptr(), rows, cols, kind, weight_kind, at, size)
    return out, grad_weight, grad_bias


def _documents(logits, tokens, row_ptr):
    """Checks logits, tokens and row_ptr; the arguments that the library's calls begin with."""
    rows, vocab, stride, kind = _rows(logits, "logits")
    device = logits.device
    n = tokens.numel() if isinstance(tokens, torch.Tensor) else -1
    at = _like(tokens, "tokens", (n,), torch.int32, device)
    if row_ptr is not None:
        at_rows = _like(row_ptr, "row_ptr", (rows + 1,), torch.int64, device)
    else:
        at_rows = 0
        if n != rows:
            raise ValueError("without row_ptr there must be one token to a row")
    return logits.data_ptr(), stride, rows, vocab, kind, at, at_rows, n


def token_logprobs(logits, tokens, row_ptr=None, alternatives: int = 0, entropy: bool = False) -> TokenLogprobs:
    """Log-probabilities of tokens (int32 words) under the softmax of their rows of logits [rows, vocab]:
    row r has the tokens row_ptr[r] .. row_ptr[r+1]-1 (int64, on the GPU, its last entry at most the number
    of tokens), or without row_ptr one each.  Tokens below zero are none.  With `alternatives` also each row's
    likeliest words, ties to the lowest; with `entropy` the entropies."""
    args = _documents(logits, tokens, row_ptr)
    rows, vocab, device = args[2], args[3], logits.device
    if not 0 <= alternatives <= min(MAX_ALTERNATIVES, vocab):
        raise ValueError(f"alternatives must be in 0 .. {min(MAX_ALTERNATIVES, vocab)}")
    logprobs, stats = _fp32(args[7], device), _fp32((rows, 2), device)
    entropies = top_ids = top_logprobs = None
    at_entropies = at_ids = at_top = 0
    if entropy:
        entropies = _fp32(rows, device)
        at_entropies = entropies.data_ptr()
    if alternatives:
        top_ids = torch.empty((rows, alternatives), dtype=torch.int32, device=device)
        top_logprobs = _fp32((rows, alternatives), device)
        at_ids, at_top = top_ids.data_ptr(), top_logprobs.data_ptr()
    size = _workspace_bytes("mlda_token_logprobs_workspace_bytes", rows, vocab, alternatives, args[4])
    held, at = _workspace(size, device)
    _launch(device, load_library().mlda_token_logprobs, *args, alternatives, logprobs.data_ptr(), stats.data_ptr(), at_entropies,
            at_ids, at_top, at, size)
    return TokenLogprobs(logprobs, stats, entropies, top_ids, top_logprobs)


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
        if entropy is None:
            raise ValueError("a gradient of the entropy needs the entropy")
        at_grad_entropy = _like(grad_entropy, "grad_entropy", (rows,), torch.float32, device)
        at_entropy = _like(entropy, "entropy", (rows,), torch.float32, device)
    if out is None:
        out = torch.empty_like(logits)
    out_stride = _rows_like(out, "out", logits)
    _launch(device, load_library().mlda_token_logprobs_backward, *args, at_stats, at_grad, at_entropy, at_grad_entropy,
            out.data_ptr(), out_stride)
    return out


def token_logprobs_grad(logits, tokens, weights, row_ptr=None, out=None):
    """A training step's loss and gradient in one: (log-probabilities of the tokens, the gradient of
    sum(weights * log-probabilities) with respect to the logits), weights [n_tokens] fp32.  `out` (logits, for
    instance) takes the gradient."""
    args = _documents(logits, tokens, row_ptr)
    device = logits.device
    at_weights = _like(weights, "weights", (args[7],), torch.float32, device)
    logprobs = _fp32(args[7], device)
    if out is None:
        out = torch.empty_like(logits)
    out_stride = _rows_like(out, "out", logits)
    size = _workspace_bytes("mlda_token_logprobs_workspace_bytes", args[2], args[3], 0, args[4])
    held, at = _workspace(size, device)
    _launch(device, load_library().mlda_token_logprobs_grad, *args, at_weights, logprobs.data_ptr(), out.data_ptr(), out_stride, at, size)
    return logprobs, out


def _tensor_list(tensors, name, device):
    """Addresses, sizes and type codes of contiguous tensors on the device, as host arrays."""
    for t in tensors:
        if not isinstance(t, torch.Tensor) or not t.is_contiguous() or t.device != device or t.dtype not in _TYPES:
            raise ValueError(f"{name} must be contiguous fp32, bf16 or fp16 tensors on one GPU")
    n = len(tensors)
    return ((ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors]), (ctypes.c_int64 * n)(*[t.numel() for t in tensors]),
            (ctypes.c_int32 * n)(*[_TYPES[t.dtype] for t in tensors]))


def _grads(tensors, max_norm, out):
    tensors = list(tensors)
    if not tensors or not isinstance(tensors[0], torch.Tensor) or not tensors[0].is_cuda:
        raise ValueError("there must be at least one tensor, on a GPU: there is no CPU path")
    n, device = len(tensors), tensors[0].device
    at, sizes, types = _tensor_list(tensors, "tensors", device)
    norm = _fp32((), device)
    size = _workspace_bytes("mlda_grad_norm_workspace_bytes", n)
    held, workspace = _workspace(size, device)
    if max_norm is None:
        _launch(device, load_library().mlda_grad_norm, at, sizes, types, n, norm.data_ptr(), workspace, size)
        return norm
    to = at
    if out is not None:
        out = list(out)
        if len(out) != n or any(o.dtype != t.dtype or o.shape != t.shape for o, t in zip(out, tensors)):
            raise ValueError("out must have a tensor of the shape and type of each of tensors")
        to = _tensor_list(out, "out", device)[0]
    _launch(device, load_library().mlda_clip_grads, at, to, sizes, types, n, max_norm, norm.data_ptr(), workspace, size)
    return norm


def grad_norm(tensors):
    """The norm over all tensors of a gradient: the square root of the sum of all squares, as a scalar
    tensor."""
    return _grads(tensors, None, None)


def clip_grads(tensors, max_norm: float, out=None):
    """Scales the tensors of a gradient, in place or into those of `out`, by max_norm / norm where their norm
    exceeds max_norm; a norm that is not finite scales nothing.  Returns the norm before."""
    return _grads(tensors, max_norm, out)
