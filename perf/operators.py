"""The operators for models that are trained and scored next to the sampled topics, as cases that can
be timed: layer norm over the topics of documents, log-probabilities of the documents' words with
their gradient, and the global gradient norm with clipping.

A case names what is done, the sizes and the types:

  "norm"       layer norm of `rows` documents over `cols` topics
  "norm_grad"  its gradients: of the input, the weight and the bias
  "score"      log-probabilities of given words out of logits over `vocab` words, the entropy of each
               row's distribution, and the `top` likeliest words
  "train"      the same log-probabilities with the gradient of their weighted sum
  "explore"    the log-probabilities and entropies first, then the gradient for given gradients of both
  "clip"       the norm over all tensors of a gradient, and the tensors scaled down to `max_norm`

`mean_len` is the documents' mean length in words (log-normal, some documents empty); 0 stands for one
word to a row, in which case there are no bounds of documents.  `masked` is the share of the
vocabulary that is not allowed (logit minus infinity).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_EPS = 1e-5


def _norm(name, rows, cols, dtype, do="norm"):
    return {"name": name, "do": do, "rows": rows, "cols": cols, "dtype": dtype}


def _words(name, do, rows, vocab, dtype, mean_len, top=0, masked=0.0):
    return {"name": name, "do": do, "rows": rows, "vocab": vocab, "dtype": dtype, "mean_len": mean_len,
            "top": top, "masked": masked}


def _clip(name, vocab, cols, tensors, dtype, max_norm=1.0):
    return {"name": name, "do": "clip", "vocab": vocab, "cols": cols, "tensors": tensors, "dtype": dtype,
            "max_norm": max_norm}


def listed():
    return [
        # One new document's thousand topics, as a server sees it: the call's own cost.
        _norm("norm_document", 1, 1000, "fp32"),
        # All documents of the news corpus at its thousand topics: one pass over 600 MB.
        _norm("norm_corpus", 300000, 1000, "bf16"),
        # A training step on the whole of the smallest benchmark corpus (32 topics).
        _norm("norm_grad_small", 1000, 32, "fp32", "norm_grad"),
        # A large batch at an odd number of topics: rows that start at odd addresses.
        _norm("norm_grad_odd", 30011, 1537, "bf16", "norm_grad"),
        # One document scored against the news vocabulary, with the alternatives that are shown to a user.
        _words("score_document", "score", 1, 102000, "bf16", 330, top=20),
        # Abstracts scored in bulk against the largest vocabulary.
        _words("score_abstracts", "score", 2048, 141000, "fp16", 90, top=5),
        # One next word for each of several thousand rows, an odd vocabulary of which a tenth is not allowed.
        _words("score_words", "score", 6007, 40009, "bf16", 0, top=20, masked=0.1),
        # A step on the smallest corpus: all of its documents, in full precision.
        _words("train_small", "train", 1000, 5000, "fp32", 100),
        # A batch of news articles: the step that training spends its time on.
        _words("train_news", "train", 1024, 102000, "bf16", 330),
        # A batch on the middle corpus, with a reward for entropy: forward and backward called apart.
        _words("explore_medium", "explore", 512, 30000, "fp32", 50),
        # The gradient of a model of the smallest corpus: a few small tensors.
        _clip("clip_small", 5000, 32, 4, "fp32"),
        # The gradient at the largest vocabulary: one very large tensor and many small ones.
        _clip("clip_large", 141000, 1000, 48, "fp32"),
    ]


def draw(rng):
    """Sizes spread over the logarithm of the listed ranges, ragged, with every type."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    do = rng.choice(["norm", "norm_grad", "score", "train", "explore", "clip"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if do in ("norm", "norm_grad"):
        cols = log_int(8, 40000)
        most = 1.2e8 if do == "norm" else 4e7
        return {"do": do, "rows": log_int(1, min(300000, most / cols)), "cols": cols, "dtype": dtype}
    if do == "clip":
        vocab = log_int(300, 141000)
        return {"do": do, "vocab": vocab, "cols": log_int(8, min(10000, 1.2e8 / vocab)), "tensors": rng.randint(1, 48),
                "dtype": dtype, "max_norm": rng.choice([0.1, 1.0, 1e9])}
    vocab = log_int(60, 141000)
    rows = log_int(1, min(20000, 1.2e8 / vocab if do == "score" else 5e7 / vocab))
    mean_len = rng.choice([0, log_int(8, min(30000, 3e6 / rows))])
    return {"do": do, "rows": rows, "vocab": vocab, "dtype": dtype, "mean_len": mean_len,
            "top": min(vocab, rng.choice([1, 5, 20])) if do == "score" else 0,
            "masked": rng.choice([0.0, 0.0, 0.1, 0.999])}


def _lengths(case):
    """The documents' lengths: of the case alone, so that every seed gives arrays of the same sizes."""
    rows = case["rows"]
    if not case["mean_len"]:
        return torch.ones(rows, dtype=torch.int64)
    normal = torch.randn(rows, generator=torch.Generator().manual_seed(rows))
    return (case["mean_len"] * torch.exp(0.5 * normal - 0.125)).floor().to(torch.int64)


def _shapes(case):
    """A word-topic matrix, its bias, and pairs of vectors and small square matrices of other layers."""
    cols, shapes = case["cols"], [(case["vocab"], case["cols"]), (case["vocab"],)]
    side = min(cols, 256)
    shapes += [[(cols,), (cols + 1,), (side, side), (7,)][i % 4] for i in range(case["tensors"])]
    return shapes[:case["tensors"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = {"case": case}
    if case["do"] in ("norm", "norm_grad"):
        rows, cols = case["rows"], case["cols"]
        x = normal(rows, cols).mul_(1.5).add_(normal(rows, 1)).to(dtype)
        state.update(x=x, weight=(1.0 + 0.2 * normal(cols)).to(dtype), bias=(0.1 * normal(cols)).to(dtype))
        if case["do"] == "norm_grad":       # what the forward pass has left
            values = x.float()
            var, mean = torch.var_mean(values, 1, unbiased=False)
            state.update(mean=mean, rstd=torch.rsqrt(var + _EPS), grad=normal(rows, cols).to(dtype))
        return state
    if case["do"] == "clip":
        state["grads"] = [(0.01 * normal(*shape)).to(dtype) for shape in _shapes(case)]
        state["clipped"] = [torch.empty_like(g) for g in state["grads"]]
        return state
    rows, vocab = case["rows"], case["vocab"]
    # words are numbered at random; a word's logit falls with the logarithm of its rank
    number = torch.randperm(vocab, generator=gen, device="cuda")
    by_rank = -1.05 * torch.log(torch.arange(1, vocab + 1, device="cuda", dtype=torch.float32))
    base = torch.empty(vocab, device="cuda")
    hidden = torch.rand(vocab, generator=gen, device="cuda") < case["masked"]
    hidden[0] = False
    base[number] = by_rank.masked_fill(hidden, -math.inf)
    state["logits"] = normal(rows, vocab).mul_(1.5).add_(base).to(dtype)
    lengths = _lengths(case)
    lengths = lengths[torch.randperm(rows, generator=torch.Generator().manual_seed(seed))]
    total = int(lengths.sum())
    rank = torch.exp(torch.rand(total, generator=gen, device="cuda") * math.log(vocab)).long().clamp_(1, vocab) - 1
    state["tokens"] = number[rank].to(torch.int32)
    state["row_ptr"] = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).cuda() if case["mean_len"] else None
    if case["do"] in ("train", "explore"):   # what each word's log-probability counts for
        state["weights"] = -(0.5 + torch.rand(total, generator=gen, device="cuda"))
    if case["do"] == "explore":
        state["entropy_weights"] = 0.01 * (0.5 + torch.rand(rows, generator=gen, device="cuda"))
    return state


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    from paper_1803_04631_amd import operators
    do = state["case"]["do"]
    if do == "norm":
        y, mean, rstd = operators.layer_norm(state["x"], state["weight"], state["bias"], _EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if do == "norm_grad":
        grad_x, grad_weight, grad_bias = operators.layer_norm_backward(
            state["grad"], state["x"], state["mean"], state["rstd"], state["weight"])
        return {"x": grad_x, "weight": grad_weight, "bias": grad_bias}
    if do == "clip":
        norm = operators.clip_grads(state["grads"], state["case"]["max_norm"], out=state["clipped"])
        return {"norm": norm, "grads": state["clipped"]}
    logits, tokens, row_ptr = state["logits"], state["tokens"], state["row_ptr"]
    if do == "score":
        r = operators.token_logprobs(logits, tokens, row_ptr, alternatives=state["case"]["top"], entropy=True)
        return {"logprobs": r.logprobs, "entropy": r.entropy, "top_ids": r.top_ids, "top_logprobs": r.top_logprobs}
    if do == "train":
        logprobs, grad = operators.token_logprobs_grad(logits, tokens, state["weights"], row_ptr)
        return {"logprobs": logprobs, "logits": grad}
    r = operators.token_logprobs(logits, tokens, row_ptr, entropy=True)
    grad = operators.token_logprobs_backward(state["weights"], logits, tokens, r.stats, row_ptr,
                                             grad_entropy=state["entropy_weights"], entropy=r.entropy)
    return {"logprobs": r.logprobs, "entropy": r.entropy, "logits": grad}


def _rows_of(row_ptr, rows, total):
    at = torch.arange(rows, device="cuda")
    return at if row_ptr is None else torch.repeat_interleave(at, row_ptr.diff(), output_size=total)


def _plain(state):
    do = state["case"]["do"]
    if do == "norm":
        x = state["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + _EPS)
        y = x * rstd[:, None] * state["weight"].float() + state["bias"].float()
        return {"y": y.to(state["x"].dtype), "mean": mean, "rstd": rstd}
    if do == "norm_grad":
        g = state["grad"].float()
        unit = (state["x"].float() - state["mean"][:, None]) * state["rstd"][:, None]
        grad_weight, grad_bias = (g * unit).sum(0), g.sum(0)
        g = g * state["weight"].float()
        grad_x = state["rstd"][:, None] * (g - g.mean(1, keepdim=True) - unit * (g * unit).mean(1, keepdim=True))
        dtype = state["x"].dtype
        return {"x": grad_x.to(dtype), "weight": grad_weight.to(dtype), "bias": grad_bias.to(dtype)}
    if do == "clip":
        most = state["case"]["max_norm"]
        norm = torch.stack([g.float().square().sum() for g in state["grads"]]).sum().sqrt()
        scale = torch.where(norm > most, most / norm, torch.ones_like(norm))
        return {"norm": norm, "grads": [(g.float() * scale).to(g.dtype) for g in state["grads"]]}
    logits, tokens = state["logits"], state["tokens"].long()
    rows, vocab = logits.shape
    row = _rows_of(state["row_ptr"], rows, len(tokens))
    x = logits.float()
    x = x - x.max(1, keepdim=True).values
    p = torch.exp(x)
    total = p.sum(1)
    logprobs = x[row, tokens] - torch.log(total)[row]
    if do in ("score", "explore"):
        p = p / total[:, None]
        entropy = torch.log(total) - torch.where(p > 0, p * x, 0.0).sum(1)
    if do == "score":
        # one whole number for a logit and its word: greater logits first, then lower words
        bits = (logits.float() + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, bits ^ 0x7fffffff, bits) << 32) - torch.arange(vocab, device="cuda")
        ids = (-torch.topk(key, state["case"]["top"], dim=1).values) & 0xffffffff
        return {"logprobs": logprobs, "entropy": entropy, "top_ids": ids.to(torch.int32),
                "top_logprobs": x.gather(1, ids) - torch.log(total)[:, None]}
    weights = state["weights"]
    if do == "train":
        p = p / total[:, None]
    summed = torch.zeros(rows, device="cuda").index_add_(0, row, weights)
    grad = -summed[:, None] * p
    if do == "explore":
        inner = torch.where(p > 0, x - torch.log(total)[:, None] + entropy[:, None], 0.0)
        grad = grad - state["entropy_weights"][:, None] * p * inner
    grad.view(-1).index_add_(0, row * vocab + tokens, weights)
    grad = grad.to(logits.dtype)
    if do == "train":
        return {"logprobs": logprobs, "logits": grad}
    return {"logprobs": logprobs, "entropy": entropy, "logits": grad}


def exact(case, seed):
    """The same in 64 bits: torch's own definitions and its differentiation of them."""
    state = prepare(case, seed)
    do = case["do"]
    if do in ("norm", "norm_grad"):
        x = state["x"].double()
        if do == "norm":
            y = torch.nn.functional.layer_norm(x, x.shape[1:], state["weight"].double(), state["bias"].double(), _EPS)
            var, mean = torch.var_mean(x, 1, unbiased=False)
            return {"y": y, "mean": mean, "rstd": 1.0 / torch.sqrt(var + _EPS)}
        # the gradients are those at the mean and deviation that are handed over, in 32 bits
        unit = (x - state["mean"].double()[:, None]) * state["rstd"].double()[:, None]
        g = state["grad"].double()
        scaled = g * state["weight"].double()
        along = scaled.mul(unit).sum(1, keepdim=True) / x.shape[1]
        grad_x = (scaled - scaled.sum(1, keepdim=True) / x.shape[1] - unit * along) * state["rstd"].double()[:, None]
        return {"x": grad_x, "weight": (g * unit).sum(0), "bias": g.sum(0)}
    if do == "clip":
        flat = [g.double().reshape(-1) for g in state["grads"]]
        norm = math.sqrt(math.fsum(float(f.dot(f)) for f in flat))
        scale = min(1.0, case["max_norm"] / norm) if norm > 0 else 1.0
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [g.double() * scale for g in state["grads"]]}
    logits = state["logits"].double().requires_grad_(do != "score")
    tokens = state["tokens"].long()
    rows, vocab = logits.shape
    row = _rows_of(state["row_ptr"], rows, len(tokens))
    logp = torch.log_softmax(logits, 1)
    logprobs = logp[row, tokens]
    if do != "train":
        entropy = -(logp.exp() * logp.clamp(min=-1e300)).sum(1)
    if do == "score":
        ids = torch.sort(state["logits"], dim=1, descending=True, stable=True).indices[:, :case["top"]]
        return {"logprobs": logprobs, "entropy": entropy, "top_ids": ids.to(torch.int32), "top_logprobs": logp.gather(1, ids)}
    weights = state["weights"].double()
    with torch.no_grad():
        p = logp.exp()
        grad = torch.zeros_like(p).index_put_((row, tokens), weights, accumulate=True)
        grad -= grad.sum(1, keepdim=True) * p
    if do == "train":
        return {"logprobs": logprobs.detach(), "logits": grad}
    by_entropy, = torch.autograd.grad((entropy * state["entropy_weights"].double()).sum(), logits)
    return {"logprobs": logprobs.detach(), "entropy": entropy.detach(), "logits": grad + by_entropy}


def work(case):
    """Every input read once, every output written once, whatever the present code moves."""
    size = 4 if case["dtype"] == "fp32" else 2
    if case["do"] == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": 2.0 * size * n + 2 * size * case["cols"] + 8 * case["rows"], "flops": 7.0 * n}
    if case["do"] == "norm_grad":
        n = case["rows"] * case["cols"]
        return {"bytes": 3.0 * size * n + 3 * size * case["cols"] + 8 * case["rows"], "flops": 13.0 * n}
    if case["do"] == "clip":
        n = float(sum(math.prod(shape) for shape in _shapes(case)))
        return {"bytes": 2 * size * n + 4, "flops": 3 * n}
    n, total = float(case["rows"] * case["vocab"]), float(_lengths(case).sum())
    bounds = 8 * (case["rows"] + 1) if case["mean_len"] else 0
    if case["do"] == "score":       # words in, their log-probabilities out, and what each row has besides
        return {"bytes": size * n + 8 * total + bounds + (4 + 8 * case["top"]) * case["rows"], "flops": 6 * n}
    if case["do"] == "train":
        return {"bytes": 2 * size * n + 12 * total + bounds, "flops": 7 * n}
    return {"bytes": 2 * size * n + 12 * total + bounds + 8 * case["rows"], "flops": 13 * n}
