"""Operators on CUDA tensors for models that are trained and scored next to the sampled topics: layer
norm, log-probabilities of documents' words with entropy and likeliest words, their gradients, and
the global gradient norm with clipping.

Argument marshalling only, like the rest of the binding (here compiled, csrc/tensors.cpp, for the sake of
small calls): everything is computed by the library's HIP kernels (include/mlda.h says what exactly),
on torch's current stream of the tensors' device, without synchronising it.  Outputs and workspaces come
from torch's allocator.  Tensors are fp32, bf16 or fp16; results are sums in fp32 or fp64 that are rounded
once.  Nothing is recorded for torch's differentiation: the backward passes are calls of their own; a tensor
that is written in place has a new version, so that torch notices where it had saved it.  A tensor
that a function does not take raises ValueError, a number that the library refuses (a negative eps, say)
MldaError, both before anything is launched.  What is written (`out`) is in an input's place where that is
said, or overlaps no input and no other output; a tensor that is clipped is listed once.

Inputs that other streams work on are the caller's to order, as with torch's own operations.
"""
from __future__ import annotations

import os
from typing import NamedTuple, Optional

import torch

from . import load_library
from ._build import TENSORS_PATH

load_library()                      # (raises where the library has not been built)
if not os.path.exists(TENSORS_PATH):
    raise ImportError(f"{TENSORS_PATH} is missing: build with a host compiler and torch's headers at hand (paper_1803_04631_amd.build())")
from . import _tensors              # noqa: E402

MAX_ALTERNATIVES = 32               # MLDA_MAX_ALTERNATIVES


class TokenLogprobs(NamedTuple):
    logprobs: torch.Tensor                     # [n_tokens] fp32
    stats: torch.Tensor                        # [rows, 2] fp32: greatest logit, ln sum exp(logit - it)
    entropy: Optional[torch.Tensor]            # [rows] fp32
    top_ids: Optional[torch.Tensor]            # [rows, alternatives] int32
    top_logprobs: Optional[torch.Tensor]       # [rows, alternatives] fp32


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None):
    """Each row of x [rows, cols] less its mean, over its standard deviation, times weight, plus bias.
    Returns (y, mean [rows], rstd [rows]); `out` (x, for instance) takes y."""
    return _tensors.layer_norm(x, weight, bias, eps, out)


def layer_norm_backward(grad_y, x, mean, rstd, weight=None, out=None):
    """(grad_x, grad_weight, grad_bias) for the gradient grad_y of layer_norm's y; the last two are of
    the weight's type (without a weight: of x's).  `out` (grad_y or x, for instance) takes grad_x."""
    return _tensors.layer_norm_backward(grad_y, x, mean, rstd, weight, out)


def token_logprobs(logits, tokens, row_ptr=None, alternatives: int = 0, entropy: bool = False) -> TokenLogprobs:
    """Log-probabilities of tokens (int32 words) under the softmax of their rows of logits [rows, vocab]:
    row r has the tokens row_ptr[r] .. row_ptr[r+1]-1 (int64, on the GPU, its last entry at most the number
    of tokens), or without row_ptr one each.  Tokens below zero are none; their log-probability is 0, and so
    is that of tokens before the first row's or behind the last row's.  With `alternatives` also each row's
    likeliest words, ties to the lowest; with `entropy` the entropies."""
    return TokenLogprobs(*_tensors.token_logprobs(logits, tokens, row_ptr, alternatives, entropy))


def token_logprobs_backward(grad_logprobs, logits, tokens, stats, row_ptr=None, grad_entropy=None, entropy=None, out=None):
    """The gradient with respect to the logits, for gradients grad_logprobs [n_tokens] of token_logprobs'
    log-probabilities and grad_entropy [rows] (with `entropy` as it came out) of its entropies.  `out` (logits, for
    instance) takes it."""
    return _tensors.token_logprobs_backward(grad_logprobs, logits, tokens, stats, row_ptr, grad_entropy, entropy, out)


def token_logprobs_grad(logits, tokens, weights, row_ptr=None, out=None):
    """A training step's loss and gradient in one: (log-probabilities of the tokens, the gradient of
    sum(weights * log-probabilities) with respect to the logits), weights [n_tokens] fp32.  `out` (logits, for
    instance) takes the gradient."""
    return _tensors.token_logprobs_grad(logits, tokens, weights, row_ptr, out)


def grad_norm(tensors):
    """The norm over all tensors of a gradient: the square root of the sum of all squares, as a scalar
    tensor."""
    return _tensors.grad_norm(tensors)


def clip_grads(tensors, max_norm: float, out=None):
    """Scales the tensors of a gradient, in place or into those of `out`, by max_norm / norm where their norm
    exceeds max_norm; a norm that is not finite scales nothing.  Returns the norm before."""
    return _tensors.clip_grads(tensors, max_norm, out)
