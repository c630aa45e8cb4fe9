"""Layer norm, log-probabilities of words and gradient clipping on the GPU, through the public entry
points, against the same in 64 bits by elementary torch operations.

Tolerances are bounds on the kernels' rounding, element by element: `u` is fp32's unit roundoff; a sum that a thread makes
term by term and lanes then join as a tree is off by at most (terms + levels) u times the sum of magnitudes; an exponential
by 4 u and its argument's rounding; a result is rounded once to its type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # (bounds of half a unit in the last place)
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_1803_04631_amd import operators
    return operators


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def close(got, want, bound, dtype=None):
    """|got - want| within the bound plus the rounding to got's type; what is not finite is the same."""
    dtype = dtype or got.dtype
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd])
    limit = bound + ROUND[dtype] * (want.abs() + bound) + TINY[dtype]
    limit = limit if isinstance(limit, torch.Tensor) else torch.full_like(want, limit)
    off = ((got - want).abs() - limit)[fine]
    assert not off.numel() or off.max().item() <= 0, f"off by {((got - want).abs() / limit)[fine].max().item():.3g} of the bound"


# ------------------------------------------------------------------------------------------ layer norm
SHAPES = [(1, 1), (1, 7), (3, 8), (5, 128), (67, 129), (130, 512), (9, 513), (33, 1000), (7, 1024), (5, 1025), (6, 2048),
          (3, 2049), (4, 4096), (3, 4097), (2, 8192), (2, 8193), (3, 16384), (2, 16385), (3, 40001)]


def norm64(x, weight, bias, eps):
    x = x.double()
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / x.shape[1] + eps)
    y = d * rstd[:, None]
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean, rstd


def check_norm(x, weight, bias, eps, got):
    y, mean, rstd = norm64(x, weight, bias, eps)
    cols = x.shape[1]
    n = 32 + cols / 1024                             # additions one after the other, and levels of the tree
    most = x.double().abs().max(1).values
    off = n * U * most                               # of the mean
    close(got[1], mean, off + U * most)
    # the variance: rounding of the sum of squares, of each deviation (once squared), and of the mean
    size = (n + 6) * U + 2 * rstd * (off + U * most) + rstd ** 2 * off ** 2
    close(got[2], rstd, rstd * (size + 4 * U))
    w = 1.0 if weight is None else weight.double().abs()
    b = 0.0 if bias is None else bias.double().abs()
    bound = w * rstd[:, None] * (off + 2 * U * most)[:, None] + (y.abs() + b) * (size + 8 * U)[:, None] + b * U
    close(got[0], y, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm(ops, shape, dtype):
    g = gen(sum(shape))
    x = (randn(g, *shape) * 1.5 + randn(g, shape[0], 1)).to(dtype)
    weight, bias = (1 + 0.3 * randn(g, shape[1])).to(dtype), randn(g, shape[1], dtype=dtype)
    check_norm(x, weight, bias, 1e-5, ops.layer_norm(x, weight, bias))
    check_norm(x, weight.float(), bias.float(), 1e-3, ops.layer_norm(x, weight.float(), bias.float(), 1e-3))
    check_norm(x, None, None, 1e-5, ops.layer_norm(x))
    check_norm(x, None, bias, 1e-5, ops.layer_norm(x, None, bias))


def norm_grad64(g, x, mean, rstd, weight):
    g, u = g.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    h = g if weight is None else g * weight.double()
    c = x.shape[1]
    dx = rstd.double()[:, None] * (h - h.sum(1, keepdim=True) / c - u * (h * u).sum(1, keepdim=True) / c)
    return dx, (g * u).sum(0), g.sum(0)


def check_norm_grad(g, x, mean, rstd, weight, got):
    dx, dw, db = norm_grad64(g, x, mean, rstd, weight)
    rows, cols = x.shape
    n = 40 + cols / 1024
    r = rstd.double()[:, None]
    x64, g64 = x.double(), g.double()
    m = mean.double()[:, None]
    h = g64.abs() if weight is None else (g64 * weight.double()).abs()
    u = (x64 - m).abs() * r
    du = 3 * U * u                                   # of u: a difference of two numbers of fp32, and a product
    mean_h, mean_hu = h.sum(1, keepdim=True) / cols, (h * u).sum(1, keepdim=True) / cols
    close(got[0], dx, r * ((h + mean_h * (1 + n) + u * mean_hu * (4 + n)) * 4 * U + 0 * du))
    terms = 60 + rows / 256                          # a team's rows one after the other, then the joins
    close(got[1], dw, (g64.abs() * u).sum(0) * (terms + 4) * U)
    close(got[2], db, g64.abs().sum(0) * terms * U)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm_backward(ops, shape, dtype):
    g = gen(sum(shape) + 1)
    x = (randn(g, *shape) * 1.5 + randn(g, shape[0], 1)).to(dtype)
    weight = (1 + 0.3 * randn(g, shape[1])).to(dtype)
    grad = randn(g, *shape, dtype=dtype)
    for w in (weight, weight.float(), None):
        _, mean, rstd = ops.layer_norm(x, w)
        check_norm_grad(grad, x, mean, rstd, w, ops.layer_norm_backward(grad, x, mean, rstd, w))


@pytest.mark.parametrize("rows,cols", [(100003, 16), (20001, 130), (5003, 1000), (3001, 1537), (1500, 2500), (700, 9000), (300, 20000)])
def test_layer_norm_many_rows(ops, rows, cols):
    g = gen(rows)
    x, grad = randn(g, rows, cols), randn(g, rows, cols)
    weight, bias = randn(g, cols), randn(g, cols)
    got = ops.layer_norm(x, weight, bias)
    check_norm(x, weight, bias, 1e-5, got)
    first = ops.layer_norm_backward(grad, x, got[1], got[2], weight)
    check_norm_grad(grad, x, got[1], got[2], weight, first)
    again = ops.layer_norm_backward(grad, x, got[1], got[2], weight)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("cols", [5, 130, 1000, 1537, 9001, 20003])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_in_place_and_in_strided_rows(ops, cols, dtype):
    g = gen(cols)
    wide = randn(g, 9, cols + 3, dtype=dtype)
    x, grad = wide[:, 1:cols + 1], randn(g, 9, cols, dtype=dtype)
    weight, bias = randn(g, cols, dtype=dtype), randn(g, cols, dtype=dtype)
    want = ops.layer_norm(x.contiguous(), weight, bias)
    before = wide.clone()
    grads = ops.layer_norm_backward(grad, x.contiguous(), want[1], want[2], weight)
    got = ops.layer_norm_backward(grad, x, want[1], want[2], weight)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    held = grad.clone()
    got = ops.layer_norm_backward(held, x, want[1], want[2], weight, out=held)
    assert got[0] is held and all(torch.equal(a, b) for a, b in zip(got, grads))
    got = ops.layer_norm(x, weight, bias, out=x)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, cols + 1:], before[:, cols + 1:])


def test_layer_norm_of_rows_that_are_hard(ops):
    g = gen(3)
    for cols in (100, 1000, 3000, 20000):
        x = randn(g, 6, cols)
        x[0] = 7.25                                  # no variance
        x[1] = 0.0
        x[2] += 30000.0                              # a mean far from zero
        x[3, 5] = NAN
        x[4, 2] = INF
        y, mean, rstd = ops.layer_norm(x)
        for i in (0, 1, 2, 5):
            check_norm(x[i:i + 1], None, None, 1e-5, (y[i:i + 1], mean[i:i + 1], rstd[i:i + 1]))
        assert (y[0] == 0).all() and torch.isnan(y[3]).all() and torch.isnan(y[4]).all()


def test_layer_norm_without_rows(ops):
    x = torch.empty(0, 300, device="cuda")
    y, mean, rstd = ops.layer_norm(x, torch.ones(300, device="cuda"))
    assert y.shape == (0, 300) and mean.shape == rstd.shape == (0,)
    grads = ops.layer_norm_backward(x, x, mean, rstd, torch.ones(300, device="cuda"))
    assert grads[0].shape == (0, 300) and not grads[1].any() and not grads[2].any()


def test_layer_norm_gradient_against_differences(ops):
    g = gen(5)
    for rows, cols in ((5, 33), (3, 700), (2, 5000)):
        x, grad, weight, bias = randn(g, rows, cols), randn(g, rows, cols), randn(g, cols), randn(g, cols)
        _, mean, rstd = ops.layer_norm(x, weight, bias)
        dx, dw, db = ops.layer_norm_backward(grad, x, mean, rstd, weight)
        to = [randn(g, *t.shape).double() for t in (x, weight, bias)]
        step = 1e-4

        def loss(s):
            return (norm64(x.double() + s * to[0], weight.double() + s * to[1], bias.double() + s * to[2], 1e-5)[0] * grad.double()).sum()

        slope = (loss(step) - loss(-step)) / (2 * step)
        parts = [(a.double() * b) for a, b in zip((dx, dw, db), to)]
        # third derivatives are of the size of the terms: step^2 of their magnitude, and fp32's rounding
        size = sum(p.abs().sum() for p in parts) + (grad.double().abs() * weight.double().abs()).sum() * 10
        assert abs(sum(p.sum() for p in parts) - slope) <= size * (step ** 2 + 200 * U)


# ------------------------------------------------------------------------------------------ log-probabilities
def documents(g, rows, vocab, total):
    """Bounds of `rows` documents, some empty, and words with repetitions."""
    cuts = torch.randint(total + 1, (rows - 1,), generator=g, device="cuda").sort().values if rows > 1 else torch.empty(0, dtype=torch.int64, device="cuda")
    row_ptr = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), total)])
    return row_ptr, torch.randint(vocab, (total,), generator=g, device="cuda", dtype=torch.int32)


def rows_of(row_ptr, rows, total):
    at = torch.arange(rows, device="cuda")
    return at if row_ptr is None else torch.repeat_interleave(at, row_ptr.diff(), output_size=total)


class Exact:
    """The definition in 64 bits.  What is not allowed has a logit of minus infinity."""

    def __init__(self, logits, tokens, row_ptr):
        x = logits.double()
        self.rows, self.vocab = x.shape
        self.x, self.tokens, self.row = x, tokens.long(), rows_of(row_ptr, self.rows, len(tokens))
        self.m = x.max(1).values
        empty = self.m == -INF
        d = x - torch.where(empty, 0.0, self.m)[:, None]
        e = torch.exp(d)
        s = e.sum(1)
        self.log_s = torch.where(empty, 0.0, torch.log(s))
        self.p = torch.where(empty[:, None], 0.0, e / s[:, None])
        self.logp = d - self.log_s[:, None]                         # (minus infinity in empty rows)
        self.entropy = torch.where(empty, 0.0, self.log_s - torch.where(e == 0, 0.0, e * d).sum(1) / s)
        self.there = (self.tokens >= 0) & (self.tokens < self.vocab)
        self.empty = empty
        at = self.tokens.clamp(0, self.vocab - 1)
        self.logprobs = torch.where(self.there, self.logp[self.row, at], torch.where(self.tokens < 0, 0.0, NAN))
        # rounding: sums of a lane's terms, exponentials, the difference to the maximum
        lane = self.vocab / 256 + 64
        self.off_log_s = (lane + 30) * U + 2 * U * (1 + self.log_s.abs())    # (of a row that allows something)
        self.off_logp = self.off_log_s[:, None] + 2 * U * self.logp.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0)
        self.spread = torch.where(empty, 0.0, torch.where(e == 0, 0.0, e * d.abs()).sum(1) / s)

    def grad(self, g, h=None):
        """The gradient and the bound of its rounding."""
        g = torch.where(self.there, g.double(), 0.0)
        flat = self.row * self.vocab + self.tokens.clamp(0, self.vocab - 1)
        own = torch.zeros(self.rows * self.vocab, dtype=torch.float64, device="cuda").index_add_(0, flat, g).view(self.rows, self.vocab)
        size = torch.zeros(self.rows * self.vocab, dtype=torch.float64, device="cuda").index_add_(0, flat, g.abs()).view(self.rows, self.vocab)
        total = own.sum(1, keepdim=True)
        inner = total.expand_as(self.p)
        off = total.abs().expand_as(self.p) * U
        if h is not None:
            part = torch.where(self.p > 0, self.logp + self.entropy[:, None], 0.0)
            inner = inner + h.double()[:, None] * part
            off = off + h.double().abs()[:, None] * (self.off_logp + 2 * U * part.abs() + (self.off_log_s * (1 + self.spread) * 4)[:, None])
        d = torch.where(self.p > 0, self.logp + self.log_s[:, None], 0.0).abs()
        relative = self.off_log_s[:, None] + (6 + 3 * d) * U
        grad = torch.where(self.empty[:, None], 0.0, own - self.p * inner)
        # exponentials below fp32's normal range may be flushed
        bound = self.p * (inner.abs() * relative + off * 2) + (size + own.abs()) * 2 * U + inner.abs() * 2.0 ** -125
        return grad, bound


def check_logprobs(ops, logits, tokens, row_ptr, alternatives, entropy=True):
    got = ops.token_logprobs(logits, tokens, row_ptr, alternatives=alternatives, entropy=entropy)
    want = Exact(logits, tokens, row_ptr)
    at = want.tokens.clamp(0, want.vocab - 1)
    off = want.off_logp[want.row, at] if len(tokens) else torch.zeros(0, dtype=torch.float64, device="cuda")
    close(got.logprobs, want.logprobs, off)
    close(got.stats[:, 0], want.m, 0.0)
    close(got.stats[:, 1], want.log_s, want.off_log_s)
    if entropy:
        close(got.entropy, want.entropy, want.off_log_s * (1 + want.spread) * 4)
    else:
        assert got.entropy is None
    if alternatives:
        ids = torch.sort(want.x + 0.0, dim=1, descending=True, stable=True).indices[:, :alternatives]
        assert torch.equal(got.top_ids.long(), ids)
        close(got.top_logprobs, want.logp.gather(1, ids), want.off_logp.gather(1, ids))
    else:
        assert got.top_ids is None and got.top_logprobs is None
    return got, want


VOCABS = [1, 2, 7, 63, 511, 2047, 2048, 2049, 8192, 8193, 16385, 40009]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs(ops, vocab, dtype):
    g = gen(vocab)
    for rows, total, top in ((1, 40, 5), (3, 0, 1), (37, 500, 20), (530, 900, 32), (530, 3000, 0)):
        if rows * vocab > 2e7:
            rows = 515
        logits = (3 * randn(g, rows, vocab)).to(dtype)
        row_ptr, tokens = documents(g, rows, vocab, total)
        check_logprobs(ops, logits, tokens, row_ptr, min(top, vocab), entropy=top != 1)
    logits = (3 * randn(g, 6, vocab)).to(dtype)
    check_logprobs(ops, logits, torch.randint(vocab, (6,), generator=g, device="cuda", dtype=torch.int32), None, min(3, vocab))


@pytest.mark.parametrize("rows", [2, 600])
@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_of_ties_orders_and_masks(ops, rows, dtype):
    g = gen(rows)
    vocab = 9001
    low = torch.finfo(dtype).min
    rank = torch.arange(vocab, device="cuda", dtype=torch.float32)
    allowed = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    allowed[[17, 4000, 4001, 8999]] = True
    base = randn(g, rows, vocab)
    cases = {
        "constant": torch.zeros(rows, vocab, device="cuda"),
        "rising": (rank / 1000).expand(rows, vocab),
        "falling": (-rank / 1000).expand(rows, vocab),
        "steps": torch.floor(rank / 500).expand(rows, vocab),
        "few values": torch.round(base),
        "both zeros": torch.where(base > 0, 0.0, -0.0) - (base > 2).float(),
        "few allowed": base.masked_fill(~allowed, -INF),
        "few allowed, lowest": base.masked_fill(~allowed, low),
        "one allowed": torch.full((rows, vocab), -INF, device="cuda").index_fill_(1, torch.tensor([123], device="cuda"), 2.0),
        "all lowest": torch.full((rows, vocab), low, device="cuda"),
        "none allowed": torch.full((rows, vocab), -INF, device="cuda"),
        "large": base * 8 + 10000,
        "wide": base * 1000,
    }
    for name, x in cases.items():
        print(name, flush=True)
        logits = x.to(dtype).contiguous()
        if name == "none allowed":
            logits[0, :] = base[0].to(dtype)
        row_ptr, tokens = documents(g, rows, vocab, 700)
        got, want = check_logprobs(ops, logits, tokens, row_ptr, 20)
        weights = randn(g, 700)
        close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr), *want.grad(weights), dtype=dtype)
        h = randn(g, rows)
        close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy),
              *want.grad(weights, h), dtype=dtype)
        logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
        assert torch.equal(logprobs.isfinite(), got.logprobs.isfinite())
        close(grad, *want.grad(weights), dtype=dtype)


@pytest.mark.parametrize("rows", [2, 600])
def test_logprobs_of_rows_with_nan_and_infinity(ops, rows):
    g = gen(rows + 1)
    vocab = 5000
    logits = randn(g, rows, vocab)
    clean = logits.clone()
    row_ptr, tokens = documents(g, rows, vocab, 900)
    row_ptr[1] = 300                                  # (a first row with words)
    row_ptr = row_ptr.cummax(0).values
    logits[0, 77] = NAN
    logits[1, 4444] = INF
    logits[1, 9] = NAN
    weights, h = randn(g, 900), randn(g, rows)
    got = ops.token_logprobs(logits, tokens, row_ptr, alternatives=20, entropy=True)
    good = ops.token_logprobs(clean, tokens, row_ptr, alternatives=20, entropy=True)
    row = rows_of(row_ptr, rows, 900)
    assert torch.isnan(got.logprobs[row < 2]).all() and torch.isnan(got.entropy[:2]).all()
    assert torch.equal(got.logprobs[row >= 2], good.logprobs[row >= 2]) and torch.equal(got.entropy[2:], good.entropy[2:])
    assert torch.isnan(got.top_logprobs[:2]).all() and torch.equal(got.top_ids[2:], good.top_ids[2:])
    key = torch.where(torch.isnan(logits), -INF, logits)                  # NaN after every number
    assert torch.equal(got.top_ids.long(), torch.sort(key, dim=1, descending=True, stable=True).indices[:, :20])
    grad = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy)
    clean_grad = ops.token_logprobs_backward(weights, clean, tokens, good.stats, row_ptr, grad_entropy=h, entropy=good.entropy)
    assert torch.isnan(grad[:2]).all() and torch.equal(grad[2:], clean_grad[2:])
    few = torch.full((1, 40), NAN, device="cuda")
    few[0, [3, 30]] = torch.tensor([-INF, 1.0], device="cuda")
    top = ops.token_logprobs(few, tokens[:1].clone().fill_(3), None, alternatives=5)
    assert top.top_ids.tolist() == [[30, 3, 0, 1, 2]] and torch.isnan(top.top_logprobs).all() and torch.isnan(top.logprobs).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,total", [(1, 1, 3), (1, 300, 0), (4, 9, 50), (3, 40009, 200), (600, 33, 4000), (520, 5001, 20000),
                                              (2, 9000, 30000), (515, 2100, 1200000), (1, 70001, 5000)])
def test_logprobs_gradients(ops, rows, vocab, total, dtype):
    g = gen(rows + vocab)
    logits = (2 * randn(g, rows, vocab)).to(dtype)
    row_ptr, tokens = documents(g, rows, vocab, total)
    weights, h = randn(g, total), randn(g, rows)
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 0)
    plain = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr)
    close(plain, *want.grad(weights))
    both = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy)
    close(both, *want.grad(weights, h))
    logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
    close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens] if total else 0.0)
    close(grad, *want.grad(weights))
    # the same bits again, and in the logits' place
    assert torch.equal(plain, ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr))
    held = logits.clone()
    assert ops.token_logprobs_backward(weights, held, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy, out=held) is held
    assert torch.equal(held, both)
    held = logits.clone()
    again = ops.token_logprobs_grad(held, tokens, weights, row_ptr, out=held)
    assert torch.equal(again[0], logprobs) and torch.equal(held, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,usual", [(30000, 300), (900, 40), (7001, 9)])
def test_logprobs_gradients_of_documents_of_very_different_lengths(ops, vocab, usual, dtype):
    """Documents that fit a workgroup's registers, its table, and neither, in one batch."""
    g = gen(vocab)
    lengths = torch.full((520,), usual, device="cuda")
    lengths[:7] = torch.tensor([8 * usual, 12 * usual, 20 * usual, 0, 1, 7 * usual, 3000], device="cuda")
    row_ptr = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    total = int(row_ptr[-1])
    logits = (2 * randn(g, 520, vocab)).to(dtype)
    tokens = torch.randint(vocab, (total,), generator=g, device="cuda", dtype=torch.int32)
    weights, h = randn(g, total), randn(g, 520)
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 3)
    close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy), *want.grad(weights, h))
    grad = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr)
    close(grad, *want.grad(weights))
    held = logits.clone()
    logprobs, _ = ops.token_logprobs_grad(held, tokens, weights, row_ptr, out=held)
    close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
    close(held, *want.grad(weights))


@pytest.mark.parametrize("rows", [5, 700])
def test_logprobs_gradients_of_one_word_a_row(ops, rows):
    g = gen(rows)
    for vocab in (1, 6, 3001):
        logits = randn(g, rows, vocab)
        tokens = torch.randint(vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        tokens[0] = -1
        weights, h = randn(g, rows), randn(g, rows)
        weights[0] = NAN                              # (of no word: counts for nothing)
        got, want = check_logprobs(ops, logits, tokens, None, 0)
        clean = torch.where(torch.isnan(weights), 0.0, weights)
        grad, bound = want.grad(clean)
        close(ops.token_logprobs_backward(weights, logits, tokens, got.stats), grad, bound)
        close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, grad_entropy=h, entropy=got.entropy), *want.grad(clean, h))
        logprobs, fused = ops.token_logprobs_grad(logits, tokens, weights)
        close(fused, grad, bound)
        assert not fused[0].any() and logprobs[0] == 0


@pytest.mark.parametrize("rows", [3, 600])
def test_words_that_are_none_or_outside_and_gradients_that_are_not_finite(ops, rows):
    g = gen(rows)
    vocab = 3001
    logits = randn(g, rows, vocab)
    total = 10 * rows
    row_ptr = torch.arange(rows + 1, device="cuda") * 10
    tokens = torch.randint(vocab, (total,), generator=g, device="cuda", dtype=torch.int32)
    tokens[3], tokens[4], tokens[5], tokens[6] = -1, vocab, 2 ** 31 - 1, -2 ** 31
    weights = randn(g, total)
    weights[3] = weights[6] = NAN
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 0)
    assert got.logprobs[3] == 0 and got.logprobs[6] == 0 and torch.isnan(got.logprobs[4:6]).all()
    clean = torch.where(torch.isnan(weights), 0.0, weights)
    for grad in (ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr), ops.token_logprobs_grad(logits, tokens, weights, row_ptr)[1]):
        close(grad, *want.grad(clean))
    for bad in (NAN, INF, -INF):
        weights[17] = bad                             # of the second row
        for grad in (ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr),
                     ops.token_logprobs_grad(logits, tokens, weights, row_ptr)[1]):
            assert torch.isnan(grad[1]).all()
            want_grad, bound = want.grad(clean)
            close(grad[2:], want_grad[2:], bound[2:])
    # gradients of very different sizes, and ones that cancel
    weights = clean * 2.0 ** torch.randint(-120, 100, (total,), generator=g, device="cuda").float()
    weights[25], tokens[25], weights[26], tokens[26] = 3e30, 7, -3e30, 7
    close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr), *Exact(logits, tokens, row_ptr).grad(weights))


def test_bounds_of_documents_are_clamped(ops):
    g = gen(8)
    for rows in (4, 600):
        logits = randn(g, rows, 700)
        tokens = torch.randint(700, (50,), generator=g, device="cuda", dtype=torch.int32)
        row_ptr = torch.full((rows + 1,), 50, device="cuda")
        row_ptr[:5] = torch.tensor([-3, 20, 10, 10 ** 12, 60], device="cuda")
        got = ops.token_logprobs(logits, tokens, row_ptr)
        # row 0: 0 .. 19; row 1: none (its end lies before its begin); row 2: 10 .. 49; the others: none
        want = Exact(logits, torch.cat([tokens[:10], tokens[10:]]), torch.tensor([0, 10] + [10] + [50] * (rows - 2), device="cuda"))
        close(got.logprobs[20:], want.logprobs[20:], want.off_logp[want.row, want.tokens][20:])
        weights = torch.ones(50, device="cuda")
        first = Exact(logits[:1], tokens[:20], None if rows == 0 else torch.tensor([0, 20], device="cuda")).grad(weights[:20])
        grad = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr)
        close(grad[:1], *first)
        assert not grad[1].any() and not grad[3:].any() and grad[2].any()


def test_logprobs_gradient_against_differences(ops):
    g = gen(11)
    for rows, vocab, total in ((2, 50, 30), (3, 5000, 100)):
        logits = randn(g, rows, vocab)
        row_ptr, tokens = documents(g, rows, vocab, total)
        weights, h, to = randn(g, total), randn(g, rows), randn(g, rows, vocab).double()
        got = ops.token_logprobs(logits, tokens, row_ptr, entropy=True)
        grad = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy)
        step = 1e-4

        def loss(s):
            e = Exact(logits.double() + s * to, tokens, row_ptr)
            return (weights.double() * e.logprobs).sum() + (h.double() * e.entropy).sum()

        slope = (loss(step) - loss(-step)) / (2 * step)
        size = (grad.double() * to).abs().sum() + (weights.abs().sum() + 20 * h.abs().sum()).double() * 10
        assert abs((grad.double() * to).sum() - slope) <= size * (step ** 2 + 200 * U)


def test_offsets_past_32_bits(ops):
    """Rows that begin more than 2^31 elements, and bytes, from the first."""
    g = gen(9)
    rows, cols, stride = 70, 1000, 2 ** 25 + 1
    wide = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((rows, cols), (stride, 1))
    x.copy_(randn(g, rows, cols, dtype=torch.bfloat16))
    y = x.contiguous()
    for a, b in zip(ops.layer_norm(x), ops.layer_norm(y)):
        assert torch.equal(a, b)
    _, mean, rstd = ops.layer_norm(y)
    grad = randn(g, rows, cols, dtype=torch.bfloat16)
    want = ops.layer_norm_backward(grad, y, mean, rstd)
    for a, b in zip(ops.layer_norm_backward(grad, x, mean, rstd), want):
        assert torch.equal(a, b)
    tokens = torch.randint(cols, (rows,), generator=g, device="cuda", dtype=torch.int32)
    weights = randn(g, rows)
    a, b = ops.token_logprobs(x, tokens, None, 4, True), ops.token_logprobs(y, tokens, None, 4, True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    want = ops.token_logprobs_grad(y, tokens, weights)[1]
    assert torch.equal(ops.token_logprobs_grad(x, tokens, weights, out=x)[1], want)


# ------------------------------------------------------------------------------------------ clipping
def check_clip(ops, tensors, max_norm):
    before = [t.clone() for t in tensors]
    size = math.sqrt(math.fsum(float((t.double() * t.double()).sum()) for t in tensors))
    out = [torch.full_like(t, 5.0) for t in tensors]
    norm = ops.clip_grads(tensors, max_norm, out=out)
    assert norm.shape == () and norm.dtype == torch.float32
    assert all(torch.equal(t, b) for t, b in zip(tensors, before))
    # (in 64 bits, then rounded: a norm beyond fp32's range comes out as infinity, though what is scaled is scaled by it)
    for got in (norm, ops.grad_norm(tensors)):
        close(got, torch.tensor(size, device="cuda").float(), 2 * U * size if size < 3e38 else 0.0)
    scale = max_norm / size if size > max_norm else 1.0
    for o, t in zip(out, tensors):
        if scale == 1.0:
            assert torch.equal(o, t)
        else:
            close(o, t.double() * scale, t.double().abs() * scale * 3 * U)
    held = ops.clip_grads(tensors, max_norm)
    assert torch.equal(held, norm) and all(torch.equal(t, o) for t, o in zip(tensors, out))


@pytest.mark.parametrize("dtype", TYPES)
def test_clip_sizes(ops, dtype):
    g = gen(1)
    for sizes in ([1], [0, 3, 0], [7, 4095, 4096, 4097, 1], [100003], [(300, 40), (300,), (40, 40, 2)], [3000000, 5], [i % 9 for i in range(250)]):
        for max_norm in (0.05, 1e9, 0.0):
            check_clip(ops, [randn(g, *(s if isinstance(s, tuple) else (s,)), dtype=dtype) for s in sizes], max_norm)


def test_clip_of_several_types_at_odd_addresses(ops):
    g = gen(2)
    tensors = [randn(g, 5001 + 100 * i, dtype=TYPES[i % 3])[1 + i % 7:] for i in range(130)]
    check_clip(ops, tensors, 1.5)


def test_clip_of_large_small_and_not_finite_gradients(ops):
    big = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), -3e38, device="cuda")]
    check_clip(ops, big, 2.0)
    check_clip(ops, [torch.full((5000,), 1e-38, device="cuda")], 1e-37)
    check_clip(ops, [torch.zeros(100, device="cuda")], 0.0)
    for bad in (NAN, INF, -INF):
        t = [torch.ones(5000, device="cuda"), torch.ones(3, device="cuda", dtype=torch.bfloat16)]
        t[0][4097] = bad
        before = [x.clone() for x in t]
        norm = ops.clip_grads(t, 0.5)
        assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(bad)
        for a, b in zip(t, before):
            assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) and torch.equal(a.isnan(), b.isnan())


# ------------------------------------------------------------------------------------------ streams and graphs
def one_step(ops, s):
    y, mean, rstd = ops.layer_norm(s["x"], s["weight"], s["bias"])
    r = ops.token_logprobs(s["logits"], s["tokens"], s["row_ptr"], alternatives=7, entropy=True)
    grad = ops.token_logprobs_backward(s["g"], s["logits"], s["tokens"], r.stats, s["row_ptr"], grad_entropy=s["h"], entropy=r.entropy)
    both = ops.token_logprobs_grad(s["logits"], s["tokens"], s["g"], s["row_ptr"])
    grads = ops.layer_norm_backward(s["x"], s["x"], mean, rstd, s["weight"])
    clipped = [torch.empty_like(t) for t in grads]
    norm = ops.clip_grads(grads, 0.5, out=clipped)
    return [y, mean, rstd, *r, grad, *both, *grads, norm, *clipped]


@pytest.mark.parametrize("rows", [7, 600])
def test_other_streams_and_graphs(ops, rows):
    def inputs(seed):
        g = gen(seed)
        row_ptr, tokens = documents(gen(77), rows, 9001, 800)
        return {"x": randn(g, rows, 1000), "weight": randn(g, 1000), "bias": randn(g, 1000), "logits": randn(g, rows, 9001), "tokens": tokens,
                "row_ptr": row_ptr, "g": randn(g, 800), "h": randn(g, rows)}

    s = inputs(1)
    want = [one_step(ops, inputs(seed)) for seed in (1, 2, 3)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = one_step(ops, s)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = one_step(ops, s)
    for i in (1, 0, 2, 1):
        for k, v in inputs(i + 1).items():
            s[k].copy_(v)
        eager = one_step(ops, inputs(i + 1))          # (the program's own work between the replays)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[i]))


# ------------------------------------------------------------------------------------------ refusals
def test_refusals(ops):
    x = torch.zeros(4, 6, device="cuda")
    v = torch.zeros(4, device="cuda")
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
    stats = torch.zeros(4, 2, device="cuda")
    good = ops.token_logprobs(x, tokens, alternatives=6)
    assert good.top_ids.shape == (4, 6)
    wrong = [
        lambda: ops.layer_norm(x.double()), lambda: ops.layer_norm(x[0]), lambda: ops.layer_norm(x.t()), lambda: ops.layer_norm(x.cpu()),
        lambda: ops.layer_norm(x[:, :0]), lambda: ops.layer_norm(x, torch.ones(5, device="cuda")), lambda: ops.layer_norm(x, torch.ones(6)),
        lambda: ops.layer_norm(x, torch.ones(6, device="cuda").half()), lambda: ops.layer_norm(x, torch.ones(6, device="cuda"), torch.ones(6, device="cuda").bfloat16()),
        lambda: ops.layer_norm(x, out=x[:3]), lambda: ops.layer_norm(x[:1].expand(4, 6)), lambda: ops.layer_norm(None),
        lambda: ops.layer_norm_backward(x[:3], x, v, v), lambda: ops.layer_norm_backward(x.half(), x, v, v), lambda: ops.layer_norm_backward(x, x, v[:3], v),
        lambda: ops.layer_norm_backward(x, x, v, v.double()), lambda: ops.layer_norm_backward(x, x, v, v, out=x.half()),
        lambda: ops.token_logprobs(x, tokens.long()), lambda: ops.token_logprobs(x, tokens[:3]), lambda: ops.token_logprobs(x, tokens.cpu()),
        lambda: ops.token_logprobs(x, tokens, tokens), lambda: ops.token_logprobs(x, tokens, torch.zeros(4, dtype=torch.int64, device="cuda")),
        lambda: ops.token_logprobs(x, tokens, alternatives=7), lambda: ops.token_logprobs(x, tokens, alternatives=-1),
        lambda: ops.token_logprobs(torch.zeros(4, 50, device="cuda"), tokens, alternatives=33), lambda: ops.token_logprobs(x.int(), tokens),
        lambda: ops.token_logprobs_backward(v[:3], x, tokens, stats), lambda: ops.token_logprobs_backward(v, x, tokens, stats[:3]),
        lambda: ops.token_logprobs_backward(v, x, tokens, stats, grad_entropy=v), lambda: ops.token_logprobs_backward(v.half(), x, tokens, stats),
        lambda: ops.token_logprobs_backward(v, x, tokens, stats, out=torch.zeros(4, 7, device="cuda")),
        lambda: ops.token_logprobs_grad(x, tokens, v.double()), lambda: ops.token_logprobs_grad(x, tokens, v[::2]),
        lambda: ops.clip_grads([], 1.0), lambda: ops.clip_grads([x.double()], 1.0), lambda: ops.clip_grads([x.t()], 1.0),
        lambda: ops.clip_grads([x, x.cpu()], 1.0), lambda: ops.clip_grads([x], 1.0, out=[]), lambda: ops.clip_grads([x], 1.0, out=[x.half()]),
        lambda: ops.grad_norm([x.cpu()]),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            print("taken:", i)
    import paper_1803_04631_amd as mlda
    for call in (lambda: ops.layer_norm(x, eps=-1.0), lambda: ops.layer_norm(x, eps=NAN), lambda: ops.clip_grads([x], -1.0), lambda: ops.clip_grads([x], NAN)):
        with pytest.raises(mlda.MldaError):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_clip_at_the_edges_of_its_units(ops, dtype):
    g = gen(21)
    for n in (8191, 8192, 8193, 16384, 16391, 8192 * 1024, 8192 * 1024 + 1):
        check_clip(ops, [randn(g, n, dtype=dtype), randn(g, 3, dtype=dtype)], 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [24001, 33001, 70001, 300001])
def test_layer_norm_of_very_long_rows(ops, cols, dtype):
    g = gen(cols)
    x = (randn(g, 3, cols) + randn(g, 3, 1)).to(dtype)
    weight, bias, grad = randn(g, cols, dtype=dtype), randn(g, cols, dtype=dtype), randn(g, 3, cols, dtype=dtype)
    got = ops.layer_norm(x, weight, bias)
    check_norm(x, weight, bias, 1e-5, got)
    check_norm_grad(grad, x, got[1], got[2], weight, ops.layer_norm_backward(grad, x, got[1], got[2], weight))
    want = ops.layer_norm_backward(grad, x, got[1], got[2], weight)[0]
    held = x.clone()
    assert torch.equal(ops.layer_norm_backward(grad, held, got[1], got[2], weight, out=held)[0], want)
    held = x.clone()
    assert torch.equal(ops.layer_norm(held, weight, bias, out=held)[0], got[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logprobs_over_millions_of_words(ops, dtype):
    g = gen(31)
    vocab = 3000017
    logits = (2 * randn(g, 2, vocab)).to(dtype)
    row_ptr, tokens = documents(g, 2, vocab, 300)
    weights, h = randn(g, 300), randn(g, 2)
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 20)
    close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy), *want.grad(weights, h))
    logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
    close(grad, *want.grad(weights))
    assert torch.equal(logprobs, got.logprobs)


@pytest.mark.parametrize("rows,vocab,inside", [(20, 300, 40), (3, 20000, 500), (600, 300, 900), (2100, 3000, 900), (520, 5001, 60), (2, 700, 9000)])
def test_tokens_of_no_row(ops, rows, vocab, inside):
    """Tokens before the first row's and behind the last row's: their log-probabilities are zeros, wherever the memory comes from."""
    g = gen(rows + inside)
    head, tail = 37, 5001
    total = head + inside + tail
    logits, weights = randn(g, rows, vocab), randn(g, total)
    row_ptr, tokens = documents(g, rows, vocab, inside)
    outside = torch.full((total,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")       # (would be NaN if they were looked up)
    outside[head:head + inside] = tokens
    want = ops.token_logprobs(logits, tokens, row_ptr).logprobs
    fused, grad = ops.token_logprobs_grad(logits, tokens, weights[head:head + inside], row_ptr)

    def used_memory():
        torch.full((total,), 5.0, device="cuda")

    for first, last in ((head, 0), (0, tail), (head, tail)):
        t, w = outside[head - first:head + inside + last], weights[head - first:head + inside + last]
        used_memory()
        got = ops.token_logprobs(logits, t, row_ptr + first).logprobs
        used_memory()
        got_fused, got_grad = ops.token_logprobs_grad(logits, t, w, row_ptr + first)
        for all_of, part in ((got, want), (got_fused, fused)):
            assert torch.equal(all_of[first:first + inside], part)
            assert not all_of[:first].any() and not all_of[first + inside:].any()
        assert torch.equal(got_grad, grad)
        assert torch.equal(ops.token_logprobs_backward(w, logits, t, ops.token_logprobs(logits, t, row_ptr + first).stats, row_ptr + first),
                           ops.token_logprobs_backward(weights[head:head + inside], logits, tokens, ops.token_logprobs(logits, tokens, row_ptr).stats, row_ptr))
    # no rows at all
    used_memory()
    got = ops.token_logprobs(logits[:0], outside, row_ptr[:1], alternatives=3, entropy=True)
    assert got.logprobs.shape == (total,) and not got.logprobs.any() and got.entropy.shape == (0,) and got.top_ids.shape == (0, 3)
    used_memory()
    logprobs, nothing = ops.token_logprobs_grad(logits[:0], outside, weights, row_ptr[:1])
    assert not logprobs.any() and nothing.shape == (0, vocab)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_gradients_of_more_columns_than_a_launch_has_groups_for(ops, dtype):
    """16 columns' sums to a workgroup of 1,024 threads: 2^25 columns would be 2^32 threads, more than a launch may have."""
    g = gen(41)
    cols = 2 ** 25 + 5
    x, grad = randn(g, 2, cols, dtype=dtype), randn(g, 2, cols, dtype=dtype)
    weight = (1 + 0.3 * randn(g, cols)).to(dtype)
    mean, rstd = x.double().mean(1).float(), (1 / x.double().std(1)).float()
    want = norm_grad64(grad, x, mean, rstd, weight)
    got = ops.layer_norm_backward(grad, x, mean, rstd, weight)
    check_norm_grad(grad, x, mean, rstd, weight, got)
    # two rows: each column's sums are two products and an addition, as far from the start as from the end
    for a, b, size in ((got[1], want[1], 6.0), (got[2], want[2], 2.0)):
        close(a, b, size * U * (grad.double().abs() * 8).sum(0))


def check_norm_grad_columns(g, x, mean, rstd, weight, got, adds):
    """The gradient of x where the sums over columns are within `adds` units of roundoff of their magnitudes.  h is rounded once and u
    twice (difference, product); a mean once more; then two differences and two products."""
    dx = norm_grad64(g, x, mean, rstd, weight)[0]
    r = rstd.double()[:, None]
    h = g.double().abs() if weight is None else (g.double() * weight.double()).abs()
    u = (x.double() - mean.double()[:, None]).abs() * r
    mean_h, mean_hu = h.sum(1, keepdim=True) / x.shape[1], (h * u).sum(1, keepdim=True) / x.shape[1]
    close(got, dx, 1.01 * r * U * (4 * h + (5 + adds) * mean_h + (9 + adds) * u * mean_hu))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [70001, 2 ** 22 + 3])
def test_layer_norm_sums_of_long_rows_lose_nothing(ops, cols, dtype):
    """Bounds that do not grow with the columns: sums are in fp64, the mean is rounded once."""
    g = gen(43)
    x = torch.empty(4, cols, device="cuda")
    x[0] = 0.1                                       # (no variance: its sum is exact in fp64)
    x[1] = 1000 + 0.5 * randn(g, cols)
    x[2] = torch.rand(cols, generator=g, device="cuda")
    x[3] = randn(g, cols)
    x = x.to(dtype)
    y, mean, rstd = ops.layer_norm(x)
    want_y, want_mean, want_rstd = norm64(x, None, None, 1e-5)
    assert not y[0].any() and torch.equal(mean[0], x[0, 0].float())
    off = (1.01 * U * want_mean.abs())               # of the mean: one rounding
    close(mean, want_mean, 0.0)
    # the deviations are rounded once, their squares' mean, eps, the root and the quotient (to an ulp, 2 u) as well
    size = 10 * U + (off * want_rstd) ** 2
    close(rstd, want_rstd, want_rstd * size)
    close(y, want_y, want_rstd[:, None] * off[:, None] + want_y.abs() * (size + 3 * U)[:, None])
    # gradients of one sign, whose sums over columns are as large as they can be
    for grad in (torch.full((4, cols), 0.1, device="cuda"), torch.rand(4, cols, generator=g, device="cuda") * 0.3 + x.float().sign()):
        grad = grad.to(dtype)
        got = ops.layer_norm_backward(grad, x, mean, rstd)
        check_norm_grad_columns(grad, x, mean, rstd, None, got[0], 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sums_over_millions_of_equal_words_lose_nothing(ops, dtype):
    """Lanes that add up thousands of equal terms each, which no exact fp32 number is: the bound is of 256 additions in fp32, however long
    the row."""
    rows, vocab, most = 512, 2 ** 21 + 11, 8192
    logits = torch.full((vocab,), -2.3, device="cuda", dtype=dtype)
    logits[:most] = 0.0                              # (every lane's maximum is the row's)
    low = float(logits[most])
    s = most + (vocab - most) * math.exp(low)
    log_s = math.log(s)
    entropy = log_s - (vocab - most) * math.exp(low) * low / s
    off = (256 + 4 + 3 * abs(low)) * U
    logits = logits.expand(rows, vocab).contiguous()
    tokens = torch.full((rows,), most + 5, device="cuda", dtype=torch.int32)
    weights = torch.full((rows,), 3.0, device="cuda")

    def all_close(got, want, bound):
        close(got, torch.full_like(got, want, dtype=torch.float64), bound)

    got = ops.token_logprobs(logits, tokens, entropy=True)
    all_close(got.stats[:, 1], log_s, off + U * log_s)
    all_close(got.logprobs, low - log_s, off + 2 * U * log_s)
    all_close(got.entropy, entropy, off * (1 + abs(low)) + U * log_s)
    fused, grad = ops.token_logprobs_grad(logits, tokens, weights, out=logits)
    all_close(fused, low - log_s, off + 2 * U * log_s)
    p = math.exp(low) / s
    all_close(grad[:, most + 6:most + 9], -3.0 * p, 3.0 * p * (off + U * log_s + 12 * U))
    all_close(grad[:, most + 5], 3.0 - 3.0 * p, 8 * U)


@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-8, 1e-20])
def test_clip_by_factors_below_the_range_of_fp32(ops, max_norm):
    """The norm is beyond fp32's range or close to its end: the factor has few bits in fp32, from 2^-150 on none, and what is scaled by it
    is still a number."""
    g = gen(51)
    large = torch.full((8195,), 3e38, device="cuda") * (1 - 0.3 * torch.rand(8195, generator=g, device="cuda"))
    for tensors in ([large], [large, large[:1000].bfloat16(), 1e30 * randn(g, 9000), randn(g, 77, dtype=torch.float16)]):
        check_clip(ops, [t.clone() for t in tensors], max_norm)
    out = [torch.empty_like(large)]
    ops.clip_grads([large], max_norm, out=out)
    # of 8,195 numbers of between 2.1e38 and 3e38 none is less than 0.7 of the largest, and their norm is max_norm
    assert float(out[0].min()) > 0.7 * max_norm / math.sqrt(8195)


def test_tensors_written_in_place_have_a_new_version(ops):
    """torch's check of tensors that it has saved for another backward pass works as with its own operations in place."""
    g = gen(61)
    x, grad, weight = randn(g, 5, 300), randn(g, 5, 300), randn(g, 300)
    tokens, weights = torch.zeros(5, dtype=torch.int32, device="cuda"), randn(g, 5)
    _, mean, rstd = ops.layer_norm(x, weight)
    stats = ops.token_logprobs(x, tokens).stats
    inputs = [x, grad, weight, tokens, weights, mean, rstd, stats]

    def writes(call, *outs):
        before = [t._version for t in (*inputs, *outs)]
        call()
        after = [t._version for t in (*inputs, *outs)]
        wanted = [b + any(t is o for o in outs) for b, t in zip(before, (*inputs, *outs))]
        assert after == wanted

    def new():
        return torch.empty_like(x)

    for out in (new(), x.clone()):
        writes(lambda: ops.layer_norm(x, weight, out=out), out)
        writes(lambda: ops.layer_norm_backward(grad, x, mean, rstd, weight, out=out), out)
        writes(lambda: ops.token_logprobs_backward(weights, x, tokens, stats, out=out), out)
        writes(lambda: ops.token_logprobs_grad(x, tokens, weights, out=out), out)
        writes(lambda: ops.clip_grads([x], 0.1, out=[out]), out)
        writes(lambda: ops.clip_grads([out, mean], 0.1), out, mean)
    writes(lambda: ops.layer_norm(x, weight))
    writes(lambda: ops.grad_norm([x, grad]))
    writes(lambda: ops.layer_norm(x, weight, out=x), x)
    writes(lambda: ops.token_logprobs_grad(x, tokens, weights, out=x), x)
    for write in (lambda y: ops.layer_norm(y, out=y), lambda y: ops.clip_grads([y], 1e-3), lambda y: ops.token_logprobs_grad(y, tokens, weights, out=y)):
        leaf = randn(g, 5, 300).requires_grad_()
        y = leaf.exp()                               # (whose derivative is y)
        write(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    with torch.inference_mode():
        y = randn(g, 5, 300)
        ops.layer_norm(y, out=y)
        ops.clip_grads([y], 0.1)


def test_clipping_wants_a_norm(ops):
    t = torch.full((10,), 3.0, device="cuda")
    out = [torch.zeros(10, device="cuda")]
    for call in (lambda: ops.clip_grads([t], None), lambda: ops.clip_grads([t], None, out=out)):
        with pytest.raises(ValueError, match="max_norm"):
            call()
    assert (t == 3.0).all() and not out[0].any()


@pytest.mark.parametrize("rows", [2, 600])
def test_probabilities_far_below_the_greatest_are_exact(ops, rows):
    """Where the difference to the greatest logit is a number of fp32, so is its exponential: three units of roundoff and those of
    the products, whatever the distance.  (A row's common factor is that of a word with the greatest logit.)"""
    vocab = 6001
    x = -80 * torch.rand(rows, vocab, generator=gen(71), device="cuda")
    x[:, :2] = 0.0
    tokens, weights = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.ones(rows, device="cuda")
    got = ops.token_logprobs(x, tokens, entropy=True)
    for grad in (ops.token_logprobs_grad(x, tokens, weights)[1], ops.token_logprobs_backward(weights, x, tokens, got.stats)):
        ratio = grad[:, 2:].double() / grad[:, 1:2].double()
        want = torch.exp(x[:, 2:].double())
        assert ((ratio / want - 1).abs().max() <= 6 * U).item(), ((ratio / want - 1).abs().max() / U).item()


# ------------------------------------------------------------------------------------------ more than the caches hold, and other forms of full size
@pytest.mark.parametrize("rows,cols,dtype", [(33001, 1537, torch.bfloat16), (33001, 1537, torch.float16), (25001, 1003, torch.float32), (6007, 9001, torch.float32),
                                             (3001, 20001, torch.bfloat16), (700, 45001, torch.float32), (1100, 50001, torch.bfloat16), (500, 70001, torch.float16)])
def test_layer_norm_of_more_than_the_caches_hold(ops, rows, cols, dtype):
    """What a call that moves more than 192 MB writes goes past the caches, by other instructions: odd rows, all forms, in place too."""
    g = gen(rows + cols)
    x = (randn(g, rows, cols) * 1.5 + randn(g, rows, 1)).to(dtype)
    grad = randn(g, rows, cols, dtype=dtype)
    assert 2 * x.numel() * x.element_size() > 192e6 or 3 * x.numel() * x.element_size() > 192e6
    for kind in {dtype, torch.float32}:
        weight, bias = (1 + 0.3 * randn(g, cols)).to(kind), randn(g, cols, dtype=kind)
        got = ops.layer_norm(x, weight, bias)
        check_norm(x, weight, bias, 1e-5, got)
        held = x.clone()
        assert torch.equal(ops.layer_norm(held, weight, bias, out=held)[0], got[0])
        grads = ops.layer_norm_backward(grad, x, got[1], got[2], weight)
        check_norm_grad(grad, x, got[1], got[2], weight, grads)
        # a lane adds up 64 columns at the most, the lanes and waves join in ten steps and 16 additions; sums in fp64 are within that, too
        check_norm_grad_columns(grad, x, got[1], got[2], weight, grads[0], 64 + 10 + 16)
        for held, args in ((x.clone(), lambda t: (grad, t)), (grad.clone(), lambda t: (t, x))):
            again = ops.layer_norm_backward(*args(held), got[1], got[2], weight, out=held)
            assert all(torch.equal(a, b) for a, b in zip(again, grads))


@pytest.mark.parametrize("rows,vocab,total,dtype", [(701, 70001, 9000, torch.bfloat16), (701, 70001, None, torch.float16), (523, 50021, 20000, torch.float32),
                                                    (523, 50021, None, torch.float32), (60, 420001, 3000, torch.float32), (9001, 5501, 90000, torch.bfloat16),
                                                    (2003, 25003, None, torch.bfloat16)])
def test_logprobs_gradients_of_more_than_the_caches_hold(ops, rows, vocab, total, dtype):
    g = gen(rows + vocab)
    logits = (2 * randn(g, rows, vocab)).to(dtype)
    assert 2 * logits.numel() * logits.element_size() > 192e6
    if total is None:
        row_ptr, tokens = None, torch.randint(vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    else:
        row_ptr, tokens = documents(g, rows, vocab, total)
    weights, h = randn(g, len(tokens)), randn(g, rows)
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 0)
    plain = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr)
    close(plain, *want.grad(weights))
    both = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy)
    close(both, *want.grad(weights, h))
    logprobs, fused = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
    close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
    close(fused, *want.grad(weights))
    del want
    for expected, call in ((plain, lambda t: ops.token_logprobs_backward(weights, t, tokens, got.stats, row_ptr, out=t)),
                           (both, lambda t: ops.token_logprobs_backward(weights, t, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy, out=t)),
                           (fused, lambda t: ops.token_logprobs_grad(t, tokens, weights, row_ptr, out=t)[1])):
        held = logits.clone()
        assert call(held) is held and torch.equal(held, expected)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logprobs_gradients_of_the_largest_table(ops, dtype):
    """Documents of about a thousand words over more columns than sums by column have room for: 8,192 slots, 96 KB of LDS.  Some fill it to
    the last word that it takes, some have one more, and are done by ranges of columns."""
    g = gen(81)
    rows, vocab = 520, 15001
    lengths = torch.randint(700, 1300, (rows,), generator=g, device="cuda")
    lengths[:8] = torch.tensor([7168, 7169, 8000, 2048, 2049, 0, 1, 20000], device="cuda")
    row_ptr = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    total = int(row_ptr[-1])
    assert total / rows > 512
    tokens = torch.randint(vocab, (total,), generator=g, device="cuda", dtype=torch.int32)
    tokens[:7168] = torch.randperm(vocab, generator=g, device="cuda")[:7168].int()       # (all different: as many slots)
    logits, weights, h = (2 * randn(g, rows, vocab)).to(dtype), randn(g, total), randn(g, rows)
    got, want = check_logprobs(ops, logits, tokens, row_ptr, 0)
    close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy), *want.grad(weights, h))
    plain = ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr)
    close(plain, *want.grad(weights))
    assert torch.equal(plain, ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr))
    logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
    close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
    close(grad, *want.grad(weights))
    held = logits.clone()
    assert torch.equal(ops.token_logprobs_grad(held, tokens, weights, row_ptr, out=held)[1], grad)


@pytest.mark.parametrize("vocab,dtype", [(1025, torch.float32), (3001, torch.bfloat16), (9001, torch.float32), (12287, torch.float32), (24571, torch.bfloat16),
                                         (20011, torch.float16)])
def test_logprobs_of_a_wave_to_a_row(ops, vocab, dtype):
    """Many rows of 4 to 48 KB: a wave walks a row of up to 24 tiles, and looks for its likeliest words by itself."""
    g = gen(vocab)
    rows = 2061
    rank = torch.arange(vocab, device="cuda", dtype=torch.float32)
    base = randn(g, rows, vocab)
    few = torch.full((vocab,), True, device="cuda")
    few[torch.randperm(vocab, generator=g, device="cuda")[:9]] = False
    row_ptr, tokens = documents(g, rows, vocab, 3 * rows)
    for name, x, top in (("random", 3 * base, 32), ("random", 3 * base, 1), ("constant", torch.zeros_like(base), 20), ("rising", (rank / 1000).expand(rows, vocab), 20),
                         ("falling", (-rank / 1000).expand(rows, vocab), 20), ("few values", torch.round(base), 5), ("nine allowed", base.masked_fill(few, -INF), 20),
                         ("nine allowed, lowest", base.masked_fill(few, torch.finfo(dtype).min), 20), ("none allowed", torch.full_like(base, -INF), 3)):
        print(name, top, flush=True)
        check_logprobs(ops, x.to(dtype).contiguous(), tokens, row_ptr, top)
    check_logprobs(ops, (3 * base).to(dtype), tokens, row_ptr, 0)
    check_logprobs(ops, (3 * base).to(dtype), tokens, row_ptr, 0, entropy=False)


def test_logprobs_of_more_rows_than_a_launch_has_groups(ops):
    g = gen(91)
    rows, vocab = 2 ** 20 + 70003, 5
    logits = randn(g, rows, vocab)
    single = torch.randint(vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    for row_ptr, tokens in ((None, single), documents(g, rows, vocab, 2 * rows)):
        weights, h = randn(g, len(tokens)), randn(g, rows)
        got, want = check_logprobs(ops, logits, tokens, row_ptr, 3)
        close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr, grad_entropy=h, entropy=got.entropy), *want.grad(weights, h))
        logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
        close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
        close(grad, *want.grad(weights))


@pytest.mark.parametrize("rows", [4, 600])
def test_words_within_clamped_bounds(ops, rows):
    """Bounds outside the tokens: the rows have the words within them, log-probabilities and gradients."""
    g = gen(rows)
    logits, tokens, weights = randn(g, rows, 700), torch.randint(700, (50,), generator=g, device="cuda", dtype=torch.int32), randn(g, 50)
    row_ptr = torch.full((rows + 1,), 10 ** 12, device="cuda")
    row_ptr[:4] = torch.tensor([-3, 20, 20, 45], device="cuda")
    good = row_ptr.clamp(0, 50)
    got, want = ops.token_logprobs(logits, tokens, row_ptr), Exact(logits, tokens, good)
    close(got.logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
    logprobs, grad = ops.token_logprobs_grad(logits, tokens, weights, row_ptr)
    close(logprobs, want.logprobs, want.off_logp[want.row, want.tokens])
    close(grad, *want.grad(weights))
    close(ops.token_logprobs_backward(weights, logits, tokens, got.stats, row_ptr), *want.grad(weights))
