"""Operators on CUDA tensors for models that are trained and scored next to the sampled topics: layer
norm, log-probabilities of documents' words with entropy and likeliest words, their gradients, the
global gradient norm with clipping, dropout, the clipped policy loss, and matrices in microscaled
4-bit floating point with the product that scores documents against them.

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


class Mx4(NamedTuple):
    """A matrix [rows, cols] held in 4 bits (include/mlda.h has the format).  Rows [a, b) of it are
    Mx4(codes[a:b], scales[a:b], cols)."""
    codes: torch.Tensor                        # [rows, 16 ceil(cols / 32)] uint8
    scales: torch.Tensor                       # [rows, ceil(cols / 32)] uint8
    cols: int


class PolicyLoss(NamedTuple):
    loss: torch.Tensor                         # scalars, fp32
    kl: torch.Tensor                           # sum of the weighted KL terms
    clipped: torch.Tensor                      # sum of the weights of the words that are clipped
    grad_logprobs: torch.Tensor                # [n_tokens] fp32: the loss' gradient


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


def mx4_quantize(x, out=None) -> Mx4:
    """x [rows, cols] in blocks of 32 columns, each with a power of two as its scale and 4 bits an element:
    the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, with a sign.  A block with NaN or infinity is NaN.
    `out` (an Mx4 of that shape) takes it."""
    return Mx4(*_tensors.mx4_quantize(x, out))


def mx4_dequantize(q: Mx4, dtype=None, out=None):
    """What q stands for, [rows, cols] of the type dtype (fp32, if neither it nor `out` says another)."""
    return _tensors.mx4_dequantize(q, dtype, out)


def mx4_linear(x, weight: Mx4, bias=None, dtype=None, out=None):
    """The product of x [rows, cols], put into 4 bits as mx4_quantize does, with the transpose of weight [words, cols], plus
    bias [words] (of the result's type, or fp32): [rows, words] of the type dtype (x's, if neither it nor `out` says
    another).  For scoring: there is no backward pass; mx4_dequantize gives the weights that one would need."""
    return _tensors.mx4_linear(x, weight, bias, dtype, out)


def dropout(x, p: float, seed: int, step=0, first_row: int = 0, residual=None, out=None):
    """x [rows, cols] with elements dropped with probability p, the others times 1 / (1 - p), plus residual.  Which ones depends on
    seed (64 bits), step and an element's row (first_row is the number of x's first) and column alone, so nothing is kept for
    the backward pass.  step: a number below 2^32, or an int64 tensor of one entry on the GPU, read when the kernel runs (a
    captured graph that counts it up draws another mask at each replay).  `out` (x or residual, for instance) takes the result."""
    return _tensors.dropout(x, p, seed, step, first_row, residual, out)


def dropout_backward(grad_y, p: float, seed: int, step=0, first_row: int = 0, out=None):
    """The gradient of dropout's x, for the gradient grad_y of its result and the same p, seed, step and first_row; that of its
    residual is grad_y itself.  `out` (grad_y, for instance) takes it."""
    return _tensors.dropout(grad_y, p, seed, step, first_row, None, out)


def policy_loss(logprobs, old_logprobs, advantages, weights=None, reference=None, row_ptr=None, low: float = 0.2, high: float = 0.2, kl: float = 0.0,
                out=None) -> PolicyLoss:
    """The clipped policy loss of words with log-probabilities logprobs [n_tokens] that were drawn with old_logprobs: the sum over
    the words of weights (1 / n_tokens each without) times -min(ratio A, clip(ratio, 1 - low, 1 + high) A), ratio = exp(logprobs -
    old_logprobs), plus kl times exp(d) - d - 1 with d = reference - logprobs (with kl = 0 a reference is only watched); and its gradient for token_logprobs_backward.  The
    advantages A are the words' own, or with row_ptr (as token_logprobs takes it) those of their rows.  A word of weight 0 and one of no row
    count for nothing, whatever their numbers are.  `out` (logprobs, for instance, but not rows' advantages) takes the gradient."""
    return PolicyLoss(*_tensors.policy_loss(logprobs, old_logprobs, advantages, weights, reference, row_ptr, low, high, kl, out))
