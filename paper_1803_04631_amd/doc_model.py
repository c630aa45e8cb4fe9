"""A log-linear model of documents' words on top of the sampled topics, trained and scored with the
operators of operators.py.

Some of each document's tokens are held out, the topics of the others are sampled, and a document's
features are the logarithms of its topic proportions.  The model is

    logits = layer_norm(features) weight^T + bias,   p(word | document) = softmax(logits)

trained by gradient descent on the tokens that were sampled, with dropout of the normed features and the
gradient's norm clipped, and scored by the log-probability of the tokens that were held out.  It can be scored with its
weights in 4 bits (DocModel.packed), and trained further to suggest words that documents do hold (suggest_words: the clipped policy loss
on words that the model has drawn itself, kept near the model as it was).  The products in 32 bits are torch's, everything
beside them the library's kernels.

    python -m paper_1803_04631_amd.doc_model docword.nytimes.txt.gz --topics 1000 --iters 50 --epochs 3 --dropout 0.1 --packed
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
    model knows those and nothing of the documents.  `dropout`: the share of the normed features that each step()
    leaves out, other ones at each step, drawn from `seed` and the step's number.  policy_step() leaves none out: its ratios are to
    log-probabilities that words were drawn with, of all features."""

    def __init__(self, n_topics: int, word_counts, device="cuda:0", dropout: float = 0.0, seed: int = 0):
        counts = torch.as_tensor(word_counts, dtype=torch.float32, device=device)
        self.scale = torch.ones(n_topics, device=device)
        self.shift = torch.zeros(n_topics, device=device)
        self.weight = torch.zeros(len(counts), n_topics, device=device)
        self.bias = torch.log((counts + 0.1) / (counts + 0.1).sum())
        self.dropout, self.seed, self.steps = dropout, seed, 0

    def _logits(self, x):
        y, mean, rstd = operators.layer_norm(x, self.scale, self.shift)
        return y, mean, rstd, torch.addmm(self.bias, y, self.weight.t())

    def _gradients(self, grad, x, y, mean, rstd, dropped: bool):
        """Gradients by weight, bias, scale and shift for a gradient of the logits; y: what was multiplied."""
        grad_y = grad @ self.weight
        if dropped:
            operators.dropout_backward(grad_y, self.dropout, self.seed, self.steps, out=grad_y)
        _, grad_scale, grad_shift = operators.layer_norm_backward(grad_y, x, mean, rstd, self.scale, out=grad_y)
        return [grad.t() @ y, grad.sum(0), grad_scale, grad_shift]

    def gradients(self, x, words: Documents):
        """(mean log-probability of the words, gradients of its negative by weight, bias, scale and shift)"""
        if self.dropout:
            y, mean, rstd = operators.layer_norm(x, self.scale, self.shift)
            operators.dropout(y, self.dropout, self.seed, self.steps, out=y)
            logits = torch.addmm(self.bias, y, self.weight.t())
        else:
            y, mean, rstd, logits = self._logits(x)
        n = max(len(words.tokens), 1)
        weights = torch.full((len(words.tokens),), -1.0 / n, device=x.device)
        logprobs, grad = operators.token_logprobs_grad(logits, words.tokens, weights, words.row_ptr, out=logits)
        return logprobs.sum() / n, self._gradients(grad, x, y, mean, rstd, self.dropout > 0)

    def _descend(self, grads, rate: float, max_norm: float):
        norm = operators.clip_grads(grads, max_norm)
        for p, g in zip((self.weight, self.bias, self.scale, self.shift), grads):
            p.sub_(g, alpha=rate)
        self.steps += 1
        return norm

    def step(self, x, words: Documents, rate: float, max_norm: float):
        """One step of gradient descent; returns (mean log-probability before it, norm of the gradient)."""
        logprob, grads = self.gradients(x, words)
        return logprob, self._descend(grads, rate, max_norm)

    def policy_gradients(self, x, words: Documents, old_logprobs, advantages, reference=None, low: float = 0.2, high: float = 0.2, kl: float = 0.0,
                         entropy: float = 0.0):
        """(operators.PolicyLoss of words that were drawn with old_logprobs, gradients of it less `entropy` times the documents' mean entropy).
        An advantage for each word."""
        y, mean, rstd, logits = self._logits(x)
        r = operators.token_logprobs(logits, words.tokens, words.row_ptr, entropy=True)
        loss = operators.policy_loss(r.logprobs, old_logprobs, advantages, reference=reference, low=low, high=high, kl=kl)
        by_entropy = torch.full((len(x),), -entropy / max(len(x), 1), device=x.device)
        grad = operators.token_logprobs_backward(loss.grad_logprobs, logits, words.tokens, r.stats, words.row_ptr, grad_entropy=by_entropy,
                                                 entropy=r.entropy, out=logits)
        return loss, self._gradients(grad, x, y, mean, rstd, False)

    def policy_step(self, x, words: Documents, old_logprobs, advantages, rate: float, max_norm: float, **how):
        """One step of gradient descent on the policy loss; returns it as it was before."""
        loss, grads = self.policy_gradients(x, words, old_logprobs, advantages, **how)
        self._descend(grads, rate, max_norm)
        return loss

    def score(self, x, words: Documents, alternatives: int = 0) -> operators.TokenLogprobs:
        """Log-probabilities of the words, the documents' entropies, and their likeliest words."""
        return operators.token_logprobs(self._logits(x)[3], words.tokens, words.row_ptr, alternatives=alternatives, entropy=True)

    def packed(self, dtype=torch.bfloat16) -> "PackedDocModel":
        """The model as it is now, for scoring, with its weights in 4 bits and logits of the type dtype.  In bf16 those are half of what a large
        product writes and what scoring reads again, and off by up to 2^-8 of themselves: 1/32 at -12, about where rare words' biases are.  With torch.float32 the
        weights and features in 4 bits are all that differs."""
        return PackedDocModel(operators.mx4_quantize(self.weight), self.bias.clone(), self.scale.clone(), self.shift.clone(), dtype)


class PackedDocModel(NamedTuple):
    """A model to score with: an eighth of the weights' bytes, and matrix instructions for 4 bits."""
    weight: operators.Mx4
    bias: torch.Tensor
    scale: torch.Tensor
    shift: torch.Tensor
    dtype: torch.dtype

    def score(self, x, words: Documents, alternatives: int = 0) -> operators.TokenLogprobs:
        y, _, _ = operators.layer_norm(x, self.scale, self.shift)
        logits = operators.mx4_linear(y, self.weight, self.bias, dtype=self.dtype)
        return operators.token_logprobs(logits, words.tokens, words.row_ptr, alternatives=alternatives, entropy=True)


def suggest_words(model: DocModel, x, documents: Documents, rounds: int, draws: int = 64, steps: int = 4, rate: float = 0.1, max_norm: float = 1.0,
                  kl: float = 0.02, seed: int = 4631, out=None):
    """Trains a model further to suggest words that the documents hold: in each round it draws `draws` words for each document, a word is worth 1
    where the document holds it, else 0, and its advantage is that less the mean; then `steps` steps on the policy loss of those
    words, with a KL term to the model as it was at first.  Prints (to `out`, or standard output) and returns rows of round, share of the drawn words that documents hold,
    KL term and clipped share of the last step."""
    if rounds < 0 or draws < 1 or steps < 1:
        raise ValueError("suggest_words: need rounds >= 0, and at least one draw and one step to each")
    rows, vocab = len(x), model.weight.shape[0]
    holds = torch.zeros(rows, vocab, dtype=torch.bool, device=x.device)
    lengths = documents.row_ptr.diff()
    holds[torch.repeat_interleave(torch.arange(rows, device=x.device), lengths, output_size=len(documents.tokens)), documents.tokens.long()] = True
    row_ptr = torch.arange(rows + 1, device=x.device) * draws
    first = model._logits(x)[3]
    generator = torch.Generator(device=x.device).manual_seed(seed)
    print("round held kl clipped", file=out)
    said = []
    for n in range(1, rounds + 1):
        logits = model._logits(x)[3]
        drawn = torch.multinomial(torch.softmax(logits, 1), draws, replacement=True, generator=generator)
        words = Documents(row_ptr, drawn.to(torch.int32).view(-1))
        old = operators.token_logprobs(logits, words.tokens, row_ptr).logprobs
        reference = operators.token_logprobs(first, words.tokens, row_ptr).logprobs
        worth = holds.gather(1, drawn).float().view(-1)
        for _ in range(steps):
            loss = model.policy_step(x, words, old, worth - worth.mean(), rate, max_norm, reference=reference, kl=kl)
        said.append((n, float(worth.mean()), float(loss.kl), float(loss.clipped)))
        print("%d %.4f %.4g %.4f" % said[-1], file=out, flush=True)
    return said


class Trained(NamedTuple):
    model: DocModel
    features: torch.Tensor         # of all documents
    seen: Documents                # the tokens that topics were sampled of, and that the model was trained on
    held: Documents                # the others
    epochs: list                   # rows of epoch, trained, held out, gradient's norm


def train(*args, **how):
    """train_documents, of which it returns the model, the features, the held-out documents and the epochs' rows."""
    t = train_documents(*args, **how)
    return t.model, t.features, t.held, t.epochs


def train_documents(doc_ptr, word_ids, V: int, K: int, iters: int, epochs: int, batch: int = 1024, rate: float = 1.0, max_norm: float = 1.0,
                    share: float = 0.2, seed: int = 4631, out=None, dropout: float = 0.0) -> Trained:
    """Samples topics of the documents' tokens but a held-out share (alpha = 50/K, beta = 0.01), trains the model on those tokens, and
    prints after each epoch (to `out`, or standard output) the mean log-probability of the tokens it was trained on and of those held out."""
    from . import Mlda
    (ptr, words), (held_ptr, held_words) = hold_out(doc_ptr, word_ids, share, seed)
    alpha = 50.0 / K
    sampler = Mlda(ptr, words, V, K, alpha, 0.01, seed)
    sampler.init_random()
    sampler.step(iters)
    x = features(*sampler.doc_topic_csr(), K, alpha)
    sampler.close()
    seen, held = Documents.on_gpu(ptr, words), Documents.on_gpu(held_ptr, held_words)
    model = DocModel(K, np.bincount(words, minlength=V), dropout=dropout, seed=seed)
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
    return Trained(model, x, seen, held, rows)


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
    ap.add_argument("--dropout", type=float, default=0.0, help="share of the features that a step of training leaves out")
    ap.add_argument("--suggest", type=int, default=0, metavar="ROUNDS", help="rounds of training on words that the model suggests for the first --batch documents")
    ap.add_argument("--packed", action="store_true", help="scores with the weights in 4 bits, and logits in bf16, at the end")
    ap.add_argument("--seed", type=int, default=4631)
    args = ap.parse_args(argv)
    doc_ptr, word_ids, V = load_docword(args.docword)
    model, x, seen, held, _ = train_documents(doc_ptr, word_ids, V, args.topics, args.iters, args.epochs, batch=args.batch, rate=args.rate, seed=args.seed,
                                              dropout=args.dropout)
    if args.suggest and len(x):
        n = min(args.batch, len(x))                    # (what is held out stays so: no word of it is rewarded)
        suggest_words(model, x[:n], seen.batch(0, n, seen.row_ptr[:n + 1].tolist()), args.suggest, seed=args.seed)
    if args.packed and len(x):
        small, bounds = model.packed(), held.row_ptr.tolist()
        both = [sum(float(m.score(x[a:a + args.batch], held.batch(a, min(a + args.batch, len(x)), bounds)).logprobs.double().sum())
                    for a in range(0, len(x), args.batch)) / max(len(held.tokens), 1) for m in (model, small)]
        print("held_out in 32 bits %.4f, in 4 bits with bf16 logits %.4f" % tuple(both))
        model = small
    n = min(args.show, len(x))
    if n:
        top = model.score(x[:n], held.batch(0, n, held.row_ptr[:n + 1].tolist()), alternatives=min(10, V))
        for d in range(n):
            print("document %d: entropy %.2f, likeliest words %s" % (d + 1, top.entropy[d], (top.top_ids[d] + 1).tolist()))


if __name__ == "__main__":
    main()
