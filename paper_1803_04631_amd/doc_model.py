"""A log-linear model of documents' words on top of the sampled topics, trained and scored with the
operators of operators.py.

Some of each document's tokens are held out, the topics of the others are sampled, and a document's
features are the logarithms of its topic proportions.  The model is

    logits = layer_norm(features) weight^T + bias,   p(word | document) = softmax(logits)

trained by gradient descent on the tokens that were sampled, with the gradient's norm clipped, and
scored by the log-probability of the tokens that were held out.  The products are torch's, everything
beside them the library's kernels.

    python -m paper_1803_04631_amd.doc_model docword.nytimes.txt.gz --topics 1000 --iters 50 --epochs 3
"""
from __future__ import annotations

import argparse
from typing import NamedTuple

import numpy as np
import torch

from . import operators


def hold_out(doc_ptr, word_ids, share: float, seed: int):
    """Splits the documents' tokens at random: ((doc_ptr, word_ids) to sample, (doc_ptr, word_ids) held out)."""
    doc_ptr, word_ids = np.asarray(doc_ptr, dtype=np.int64), np.asarray(word_ids, dtype=np.int32)
    held = np.random.default_rng(seed).random(len(word_ids)) < share
    before = np.concatenate([[0], np.cumsum(held)])[doc_ptr]
    return (doc_ptr - before, word_ids[~held]), (before, word_ids[held])


class Documents(NamedTuple):
    """Documents' words on the GPU, row by row of a batch."""
    row_ptr: torch.Tensor          # int64 [documents + 1]
    tokens: torch.Tensor           # int32

    @classmethod
    def on_gpu(cls, doc_ptr, word_ids, device="cuda:0"):
        return cls(torch.as_tensor(doc_ptr, dtype=torch.int64, device=device), torch.as_tensor(word_ids, dtype=torch.int32, device=device))

    def batch(self, first: int, last: int, bounds):
        """The documents [first, last); `bounds`: row_ptr on the host."""
        a, b = int(bounds[first]), int(bounds[last])
        return Documents(self.row_ptr[first:last + 1] - a, self.tokens[a:b])


def features(row_ptr, topics, counts, n_topics: int, alpha: float, device="cuda:0"):
    """Logarithms of the documents' topic proportions, [documents, topics], out of the rows that
    Mlda.doc_topic_csr gives."""
    row_ptr = torch.as_tensor(row_ptr, device=device)
    rows = len(row_ptr) - 1
    x = torch.full((rows, n_topics), alpha, device=device)
    row = torch.repeat_interleave(torch.arange(rows, device=device), row_ptr.diff(), output_size=len(topics))
    x[row, torch.as_tensor(topics.astype(np.int64), device=device)] += torch.as_tensor(counts, dtype=torch.float32, device=device)
    return x.div_(x.sum(1, keepdim=True)).log_()


class DocModel:
    """The model's parameters, fp32.  The bias starts at the words' frequencies, so that the untrained
    model knows those and nothing of the documents."""

    def __init__(self, n_topics: int, word_counts, device="cuda:0"):
        counts = torch.as_tensor(word_counts, dtype=torch.float32, device=device)
        self.scale = torch.ones(n_topics, device=device)
        self.shift = torch.zeros(n_topics, device=device)
        self.weight = torch.zeros(len(counts), n_topics, device=device)
        self.bias = torch.log((counts + 0.1) / (counts + 0.1).sum())

    def _logits(self, x):
        y, mean, rstd = operators.layer_norm(x, self.scale, self.shift)
        return y, mean, rstd, torch.addmm(self.bias, y, self.weight.t())

    def gradients(self, x, words: Documents):
        """(mean log-probability of the words, gradients of its negative by weight, bias, scale and shift)"""
        y, mean, rstd, logits = self._logits(x)
        n = max(len(words.tokens), 1)
        weights = torch.full((len(words.tokens),), -1.0 / n, device=x.device)
        logprobs, grad = operators.token_logprobs_grad(logits, words.tokens, weights, words.row_ptr, out=logits)
        grad_y = grad @ self.weight
        _, grad_scale, grad_shift = operators.layer_norm_backward(grad_y, x, mean, rstd, self.scale, out=grad_y)
        return logprobs.sum() / n, [grad.t() @ y, grad.sum(0), grad_scale, grad_shift]

    def step(self, x, words: Documents, rate: float, max_norm: float):
        """One step of gradient descent; returns (mean log-probability before it, norm of the gradient)."""
        logprob, grads = self.gradients(x, words)
        norm = operators.clip_grads(grads, max_norm)
        for p, g in zip((self.weight, self.bias, self.scale, self.shift), grads):
            p.sub_(g, alpha=rate)
        return logprob, norm

    def score(self, x, words: Documents, alternatives: int = 0) -> operators.TokenLogprobs:
        """Log-probabilities of the words, the documents' entropies, and their likeliest words."""
        return operators.token_logprobs(self._logits(x)[3], words.tokens, words.row_ptr, alternatives=alternatives, entropy=True)


def train(doc_ptr, word_ids, V: int, K: int, iters: int, epochs: int, batch: int = 1024, rate: float = 1.0, max_norm: float = 1.0,
          share: float = 0.2, seed: int = 4631, out=None):
    """Samples topics of the documents' tokens but a held-out share (alpha = 50/K, beta = 0.01), trains the model on those tokens, and
    prints after each epoch (to `out`, or standard output) the mean log-probability of the tokens it was trained on and of those held out.  Returns (the
    model, the features, the held-out documents, rows of epoch, trained, held out, gradient's norm)."""
    from . import Mlda
    (ptr, words), (held_ptr, held_words) = hold_out(doc_ptr, word_ids, share, seed)
    alpha = 50.0 / K
    sampler = Mlda(ptr, words, V, K, alpha, 0.01, seed)
    sampler.init_random()
    sampler.step(iters)
    x = features(*sampler.doc_topic_csr(), K, alpha)
    sampler.close()
    seen, held = Documents.on_gpu(ptr, words), Documents.on_gpu(held_ptr, held_words)
    model = DocModel(K, np.bincount(words, minlength=V))
    batches = [(first, min(first + batch, len(ptr) - 1)) for first in range(0, len(ptr) - 1, batch)]

    def held_out():
        parts = [model.score(x[a:b], held.batch(a, b, held_ptr)).logprobs.double().sum() for a, b in batches]
        return float(torch.stack(parts).sum()) / max(len(held_words), 1)

    rows = [(0, float("nan"), held_out(), float("nan"))]
    print("epoch trained held_out norm", file=out)
    print("%d %.4f %.4f %.3g" % rows[0], file=out, flush=True)
    for epoch in range(1, epochs + 1):
        steps = [model.step(x[a:b], seen.batch(a, b, ptr), rate, max_norm) for a, b in batches]
        logprob, norm = torch.stack([torch.stack(s) for s in steps]).mean(0).tolist()
        rows.append((epoch, logprob, held_out(), norm))
        print("%d %.4f %.4f %.3g" % rows[-1], file=out, flush=True)
    return model, x, held, rows


def main(argv=None):
    from .bow import load_docword
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("docword", help="docword.*.txt or .txt.gz")
    ap.add_argument("--topics", type=int, default=1000)
    ap.add_argument("--iters", type=int, default=50, help="iterations of the sampler")
    ap.add_argument("--epochs", type=int, default=3)
    ap.add_argument("--batch", type=int, default=1024, help="documents of a step")
    ap.add_argument("--rate", type=float, default=1.0)
    ap.add_argument("--show", type=int, default=3, help="documents whose likeliest words are printed at the end")
    ap.add_argument("--seed", type=int, default=4631)
    args = ap.parse_args(argv)
    doc_ptr, word_ids, V = load_docword(args.docword)
    model, x, held, _ = train(doc_ptr, word_ids, V, args.topics, args.iters, args.epochs, batch=args.batch, rate=args.rate, seed=args.seed)
    n = min(args.show, len(x))
    if n:
        bounds = held.row_ptr[:n + 1].tolist()
        top = model.score(x[:n], held.batch(0, n, bounds), alternatives=min(10, V))
        for d in range(n):
            print("document %d: entropy %.2f, likeliest words %s" % (d + 1, top.entropy[d], (top.top_ids[d] + 1).tolist()))


if __name__ == "__main__":
    main()
