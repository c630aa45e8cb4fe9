"""More operators for models that are trained and scored next to the sampled topics, as cases that can be
timed: word matrices in microscaled 4-bit floating point and the product with them, dropout whose mask is
drawn from a counter and never stored, and the clipped policy loss between log-probabilities and their gradient.

A case names what is done, the sizes and the types:

  "pack"       a matrix of `rows` x `cols` into 4 bits and back: what the packed matrix stands for
  "linear"     the product of `rows` documents' `cols` features, put into 4 bits on the way, with a word matrix of
               `words` rows that is held in 4 bits, plus a bias: logits of the features' type
  "dropout"    dropout of `rows` x `cols` elements with probability `p`; with `residual` added to another matrix
  "dropout_grad"  its gradient
  "policy"     loss, KL term, clipped share and gradient for the log-probabilities of documents' words;
               `mean_len` is the mean length (log-normal, some documents empty) and each document has one advantage;
               0: `rows` words with an advantage each.  `kl`: the weight of the KL term, 0 without a reference

In 4 bits a row is cut into blocks of 32 columns.  A block's scale is the least power of two, from 2^-127 on, of
which seven times exceed the block's greatest magnitude; its elements are divided by it and rounded (ties to even)
to 0, 0.5, 1, 1.5, 2, 3, 4 or 6 with a sign.  Element 2j is the lower half of byte j of the codes, whose rows are
filled up with zeros to whole blocks; scales are bytes, the exponent plus 127, and 255 for a block with NaN or infinity.

An element of dropout is kept where a 32-bit number is at least p 2^32.  Its upper half is the element's 16 bits of Philox4x32-10
with the seed as key and the counter (column / 8, row, step, 1), two elements to a word, the even column's lower; its
lower half is the same of the counter (column / 8, row, step, 2).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_LOW, _HIGH = 0.2, 0.25
_U32 = 0xffffffff


def _pack(name, rows, cols, dtype):
    return {"name": name, "do": "pack", "rows": rows, "cols": cols, "dtype": dtype}


def _linear(name, rows, cols, words, dtype):
    return {"name": name, "do": "linear", "rows": rows, "cols": cols, "words": words, "dtype": dtype}


def _dropout(name, do, rows, cols, dtype, p, residual=False):
    return {"name": name, "do": do, "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _policy(name, rows, mean_len, kl):
    return {"name": name, "do": "policy", "rows": rows, "mean_len": mean_len, "kl": kl}


def listed():
    return [
        # The word matrix of the smallest benchmark corpus, in full precision.
        _pack("pack_small", 5000, 32, "fp32"),
        # The largest vocabulary's word matrix at a thousand topics, as it leaves training.
        _pack("pack_large", 141000, 1000, "fp32"),
        # One new document against the largest vocabulary, as a server sees it: the weights are what is read.
        _linear("linear_document", 1, 1000, 141000, "fp32"),
        # A few documents that arrive together, odd sizes: a last block of one column, words at odd addresses.
        _linear("linear_few", 17, 1537, 40009, "fp16"),
        # All documents of the smallest corpus at its 32 topics: a single block to a row.
        _linear("linear_small", 1000, 32, 5000, "fp32"),
        # Abstracts scored in bulk against the largest vocabulary.
        _linear("linear_abstracts", 2048, 1000, 141000, "bf16"),
        # One document's features: the call's own cost.
        _dropout("dropout_document", "dropout", 1, 1000, "fp32", 0.1),
        # Normed features of all documents of the news corpus, added to what bypasses them.
        _dropout("dropout_corpus", "dropout", 300000, 1000, "bf16", 0.1, residual=True),
        # The gradient at an odd number of topics, half of them dropped.
        _dropout("dropout_grad_odd", "dropout_grad", 30011, 1537, "bf16", 0.5),
        # One document's words.
        _policy("policy_document", 1, 330, 0.05),
        # A batch of news articles, each with one advantage, kept near a reference.
        _policy("policy_news", 1024, 330, 0.05),
        # All words of a large batch of rollouts, an advantage to each word, without a reference.
        _policy("policy_words", 50000007, 0, 0.0),
    ]


def draw(rng):
    """Sizes spread over the logarithm of the listed ranges, ragged, with every type."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    do = rng.choice(["pack", "linear", "linear", "dropout", "dropout_grad", "policy"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if do == "pack":
        cols = log_int(8, 10000)
        return {"do": do, "rows": log_int(1, min(141000, 1.2e8 / cols)), "cols": cols, "dtype": dtype}
    if do == "linear":
        words, cols = log_int(60, 141000), log_int(8, 10000)
        cols = min(cols, int(1.2e8 / words))
        return {"do": do, "rows": log_int(1, min(4096, 2.5e8 / words, 5e11 / (2.0 * words * cols))), "cols": cols, "words": words, "dtype": dtype}
    if do == "policy":
        mean_len = rng.choice([0, log_int(8, 3000)])
        return {"do": do, "rows": log_int(1, 4e7 / max(mean_len, 1)), "mean_len": mean_len, "kl": rng.choice([0.0, 0.02])}
    cols = log_int(8, 40000)
    return {"do": do, "rows": log_int(1, min(300000, 1.2e8 / cols)), "cols": cols, "dtype": dtype, "p": rng.choice([0.0, 0.1, 0.3, 0.5]),
            "residual": do == "dropout" and rng.random() < 0.5}


def _lengths(case):
    """The documents' lengths: of the case alone, so that every seed gives arrays of the same sizes."""
    normal = torch.randn(case["rows"], generator=torch.Generator().manual_seed(case["rows"]))
    return (case["mean_len"] * torch.exp(0.5 * normal - 0.125)).floor().to(torch.int64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES.get(case.get("dtype"))
    do = case["do"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = {"case": case}
    if do == "pack":        # topics weigh differently
        state["x"] = normal(case["rows"], case["cols"]).mul_(0.05 * torch.exp(0.5 * normal(case["cols"]))).to(dtype)
    elif do == "linear":
        words, cols = case["words"], case["cols"]
        weight = normal(words, cols).mul_(0.05 * torch.exp(0.5 * normal(cols)))
        codes, scales = _codes(weight)
        by_rank = -1.05 * torch.log(torch.arange(1, words + 1, device="cuda", dtype=torch.float32))
        state.update(x=normal(case["rows"], cols).to(dtype), codes=codes, scales=scales, bias=by_rank[torch.randperm(words, generator=gen, device="cuda")])
    elif do in ("dropout", "dropout_grad"):
        state["x"] = normal(case["rows"], case["cols"]).to(dtype)
        state["residual"] = normal(case["rows"], case["cols"]).to(dtype) if case["residual"] else None
        state["seed"], state["step"] = 4631 + (seed << 20), 100 + seed % 1000
    else:
        if case["mean_len"]:
            lengths = _lengths(case)[torch.randperm(case["rows"], generator=torch.Generator().manual_seed(seed))]
            n = int(lengths.sum())
            state["row_ptr"] = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).cuda()
        else:
            n = case["rows"]
            state["row_ptr"] = None
        # words as they were drawn; the model has moved a little since, and further from the reference
        old = -torch.rand(n, generator=gen, device="cuda").mul_(math.log(141000.0))
        state.update(old=old, logprobs=old + 0.2 * normal(n), reference=old + 0.4 * normal(n) if case["kl"] else None, advantages=normal(case["rows"]))
        used = torch.rand(n, generator=gen, device="cuda") >= 0.05    # words that do not count weigh nothing
        state["weights"] = used.float() / max(n, 1)
    return state


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    from paper_1803_04631_amd import operators
    case = state["case"]
    do = case["do"]
    if do == "pack":
        return {"values": operators.mx4_dequantize(operators.mx4_quantize(state["x"]))}
    if do == "linear":
        weight = operators.Mx4(state["codes"], state["scales"], case["cols"])
        return {"logits": operators.mx4_linear(state["x"], weight, state["bias"])}
    if do == "dropout":
        return {"y": operators.dropout(state["x"], case["p"], state["seed"], state["step"], residual=state["residual"])}
    if do == "dropout_grad":
        return {"x": operators.dropout_backward(state["x"], case["p"], state["seed"], state["step"])}
    r = operators.policy_loss(state["logprobs"], state["old"], state["advantages"], state["weights"], reference=state["reference"],
                              row_ptr=state["row_ptr"], low=_LOW, high=_HIGH, kl=case["kl"])
    return {"loss": r.loss, "kl": r.kl, "clipped": r.clipped, "logprobs": r.grad_logprobs}


def _blocks(x):
    """A matrix in 32 bits, cut into blocks, and the exponents of their scales (128: NaN or infinity in the block)."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 32)).view(x.shape[0], -1, 32)
    bits = x.abs().amax(2).view(torch.int32)
    exponent = ((bits >> 23) - 129 + ((bits & 0x7fffff) >= 0x600000).int()).clamp(min=-127)
    finite = torch.isfinite(x).all(2)
    return x, torch.where(finite, exponent, 128)


def _rounded(x, exponent):
    """The blocks' elements over their scales, rounded to what 4 bits hold."""
    m = x * ((127 - exponent) << 23).view(torch.float32)[:, :, None]
    a = m.abs()
    a = torch.where(a < 2, (2 * a).round() / 2, torch.where(a < 4, a.round(), 2 * (a / 2).round()))
    return torch.copysign(a, m)


def _power(exponent):
    """2 to the power of -127 .. 126, in 32 bits."""
    return torch.where(exponent == -127, 1 << 22, (exponent + 127) << 23).to(torch.int32).view(torch.float32)


def _values(x):
    """What the blocks of a matrix stand for, [rows, columns filled up to whole blocks], in 32 bits."""
    blocks, exponent = _blocks(x)
    bad = exponent == 128
    exponent = exponent.masked_fill(bad, 0)
    values = (_rounded(blocks, exponent) * _power(exponent)[:, :, None]).masked_fill(bad[:, :, None], math.nan)
    return values.view(x.shape[0], -1)


def _codes(x):
    """A matrix held in 4 bits: (codes, scales), both bytes."""
    blocks, exponent = _blocks(x)
    bad = exponent == 128
    v = _rounded(blocks, exponent.masked_fill(bad, 0))
    a = v.abs()
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, 0.5 * a + 4)).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    code = code.masked_fill(bad[:, :, None], 0).view(x.shape[0], -1, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, (exponent + 127).to(torch.uint8)


def _unpacked(codes, scales):
    """What codes and scales stand for, in 32 bits."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    values = table[torch.stack([codes & 15, codes >> 4], 2).int()].view(codes.shape[0], -1, 32)
    scale = torch.where(scales == 255, math.nan, _power((scales.int() - 127).clamp(max=126)))
    return (values * scale[:, :, None]).view(codes.shape[0], -1)


def _philox(c, key):
    """Philox4x32-10 of four counter words in 64 bits each: ten rounds, the key moving on between them."""
    k0, k1 = key & _U32, key >> 32 & _U32
    c0, c1, c2, c3 = c
    for i in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57         # modulo 2^64
        k = (k0 + i * 0x9E3779B9) & _U32, (k1 + i * 0xBB67AE85) & _U32
        c0, c1, c2, c3 = (b >> 32 & _U32) ^ c1 ^ k[0], b & _U32, (a >> 32 & _U32) ^ c3 ^ k[1], a & _U32
    return c0, c1, c2, c3


def _sixteen(rows, cols, seed, step, which):
    """The 16 bits of each element, [rows, cols]."""
    at = torch.arange((cols + 7) // 8, device="cuda")[None, :]
    row = torch.arange(rows, device="cuda")[:, None]
    words = torch.stack(torch.broadcast_tensors(*_philox((at, row, torch.full_like(at, step), torch.full_like(at, which)), seed)), 2)
    return torch.stack([words & 0xffff, words >> 16], 3).to(torch.int32).view(rows, -1)[:, :cols]


def _plain(state):
    case = state["case"]
    do = case["do"]
    if do == "pack":
        return {"values": _values(state["x"])[:, :case["cols"]].contiguous()}
    if do == "linear":
        weight = _unpacked(state["codes"], state["scales"])
        return {"logits": (_values(state["x"]) @ weight.t() + state["bias"]).to(state["x"].dtype)}
    if do in ("dropout", "dropout_grad"):
        x = state["x"]
        size = x.shape[0], x.shape[1], state["seed"], state["step"]
        number = _sixteen(*size, 1).long() << 16 | _sixteen(*size, 2)
        y = torch.where(number >= round(case["p"] * 2.0 ** 32), x.float() * (1.0 / (1.0 - case["p"])), 0.0)
        if state["residual"] is not None:
            y = y + state["residual"].float()
        return {"y" if do == "dropout" else "x": y.to(x.dtype)}
    # borders and differences of like exponentials: 64 bits
    l, o, w = state["logprobs"].double(), state["old"].double(), state["weights"].double()
    a = state["advantages"].double()
    if state["row_ptr"] is not None:
        a = torch.repeat_interleave(a, state["row_ptr"].diff(), output_size=len(l))
    d = l - o
    ratio = torch.exp(d)
    over, under = (a > 0) & (d > math.log1p(_HIGH)), (a < 0) & (d < math.log1p(-_LOW))
    clipped = over | under
    loss = -torch.where(over, 1.0 + _HIGH, torch.where(under, 1.0 - _LOW, ratio)) * a
    grad = torch.where(clipped, 0.0, -ratio * a)
    kl = torch.zeros((), dtype=torch.float64, device="cuda")
    if state["reference"] is not None:
        e = state["reference"].double() - l
        term = torch.expm1(e) - e
        kl = (w * term).sum()
        loss = loss + case["kl"] * term
        grad = grad - case["kl"] * torch.expm1(e)
    return {"loss": (w * loss).sum().float(), "kl": kl.float(), "clipped": (w * clipped).sum().float(), "logprobs": (w * grad).float()}


def _exact_values(x):
    """What 4 bits hold of a matrix, by looking for the nearest of their numbers."""
    rows, cols = x.shape
    blocks = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    blocks[:, :cols] = x
    blocks = blocks.view(rows, -1, 32)
    most = blocks.abs().amax(2, keepdim=True)
    fraction, exponent = torch.frexp(most / 7.0)                # most < 7 * 2^exponent, and not less than 7 * 2^(exponent - 1)
    exponent = torch.where(most > 0, exponent, -127).clamp(min=-127).double()
    scale = torch.exp2(exponent)
    scale = torch.where(most >= 7.0 * scale, 2.0 * scale, torch.where((most < 3.5 * scale) & (exponent > -127), 0.5 * scale, scale))
    m = blocks.abs() / scale
    # from each number to the next one at the middle between them; an even one keeps the middle itself
    held = torch.zeros_like(m)
    for middle, step, keeps in ((0.25, 0.5, True), (0.75, 0.5, False), (1.25, 0.5, True), (1.75, 0.5, False), (2.5, 1.0, True), (3.5, 1.0, False), (5.0, 2.0, True)):
        held += step * (m > middle if keeps else m >= middle)
    return (torch.sign(blocks) * held * scale).view(rows, -1)


def _exact_kept(case, state):
    """Which elements dropout keeps, with products of 16-bit halves."""
    rows, cols = case["rows"], case["cols"]
    most = round(case["p"] * 2 ** 32)

    def high_low(x, m):
        x0, x1, m0, m1 = x & 0xffff, x >> 16, m & 0xffff, m >> 16
        low = x0 * m0
        middle = x1 * m0 + (low >> 16)
        other = x0 * m1 + (middle & 0xffff)
        return x1 * m1 + (middle >> 16) + (other >> 16), (other & 0xffff) << 16 | low & 0xffff

    def numbers(row, group, which):
        c = [group, row, torch.full_like(row, state["step"]), torch.full_like(row, which)]
        k = [state["seed"] % 2 ** 32, state["seed"] // 2 ** 32 % 2 ** 32]
        for _ in range(10):
            (h0, l0), (h2, l2) = high_low(c[0], 0xD2511F53), high_low(c[2], 0xCD9E8D57)
            c = [h2 ^ c[1] ^ k[0], l2, h0 ^ c[3] ^ k[1], l0]
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        return torch.stack(c, -1)

    kept = torch.empty(rows, cols, dtype=torch.bool, device="cuda")
    for first in range(0, rows, 50000):
        row, group = torch.meshgrid(torch.arange(first, min(first + 50000, rows), device="cuda"), torch.arange(-(-cols // 8), device="cuda"), indexing="ij")
        words = numbers(row.contiguous(), group.contiguous(), 1)
        upper = torch.empty(*words.shape, 2, dtype=torch.int32, device="cuda")
        upper[..., 0], upper[..., 1] = words % 65536, words // 65536
        upper = upper.view(len(row), -1)[:, :cols]
        part = upper > most >> 16
        r, c = (upper == most >> 16).nonzero(as_tuple=True)
        lower = numbers(r + first, c // 8, 2).gather(1, (c % 8 // 2)[:, None])[:, 0] // torch.where(c % 2 == 1, 65536, 1) % 65536
        part[r, c] = lower >= most % 65536
        kept[first:first + len(row)] = part
    return kept


def exact(case, seed):
    state = prepare(case, seed)
    do = case["do"]
    if do == "pack":
        return {"values": _exact_values(state["x"])[:, :case["cols"]].contiguous()}
    if do == "linear":
        codes, cols = state["codes"].long(), state["codes"].shape[1] * 2
        half = torch.empty(*state["codes"].shape, 2, dtype=torch.int64, device="cuda")
        half[..., 0], half[..., 1] = codes % 16, codes // 16
        size = half % 8
        value = torch.where(size < 2, 0.5 * size, (1 + 0.5 * (size % 2)) * torch.exp2((size // 2).double() - 1))
        value = torch.where(half >= 8, -value, value).view(-1, cols // 32, 32)
        weight = (value * torch.exp2(state["scales"].double() - 127.0)[:, :, None]).view(-1, cols)
        del half, size, value, codes
        return {"logits": torch.addmm(state["bias"].double(), _exact_values(state["x"]), weight.t())}
    if do in ("dropout", "dropout_grad"):
        y = state["x"].double() / (1.0 - case["p"])
        y[~_exact_kept(case, state)] = 0.0
        if state["residual"] is not None:
            y += state["residual"].double()
        return {"y" if do == "dropout" else "x": y}
    l = state["logprobs"].double().requires_grad_()
    ratio = torch.exp(l - state["old"].double())
    a, w = state["advantages"].double(), state["weights"].double()
    if state["row_ptr"] is not None:
        a = a[torch.searchsorted(state["row_ptr"][1:], torch.arange(len(w), device="cuda"), right=True)]
    bounded = ratio.clamp(1.0 - _LOW, 1.0 + _HIGH)
    loss = -torch.minimum(ratio * a, bounded * a)
    clipped = bounded * a < ratio * a
    kl = torch.zeros((), dtype=torch.float64, device="cuda")
    if state["reference"] is not None:
        x = state["reference"].double() - l
        term = torch.exp(x) - x - 1.0
        kl = (w * term).sum()
        loss = loss + case["kl"] * term
    loss = (w * loss).sum()
    grad, = torch.autograd.grad(loss, l)
    # where a word is not clipped both arguments of the minimum are one number, and each has half of the gradient
    return {"loss": loss.detach(), "kl": kl.detach(), "clipped": w[clipped].sum(), "logprobs": grad}


def work(case):
    """Every input read once, every output written once, whatever the present code moves."""
    size = {"fp32": 4, "bf16": 2, "fp16": 2}.get(case.get("dtype"), 4)
    if case["do"] == "pack":        # the packed matrix is written, and read for the values
        n, packed = float(case["rows"] * case["cols"]), 17.0 * case["rows"] * -(-case["cols"] // 32)
        return {"bytes": (size + 4) * n + 2 * packed, "flops": 4 * n}
    if case["do"] == "linear":
        rows, cols, words = float(case["rows"]), case["cols"], case["words"]
        return {"bytes": size * rows * (cols + words) + 17.0 * words * -(-cols // 32) + 4 * words, "flops": 2 * rows * cols * words}
    if case["do"] in ("dropout", "dropout_grad"):
        n = float(case["rows"] * case["cols"])
        return {"bytes": (3 if case["residual"] else 2) * size * n, "flops": 2 * n}
    n = float(_lengths(case).sum()) if case["mean_len"] else float(case["rows"])
    each = 4 * n if not case["mean_len"] else 12 * case["rows"] + 8
    return {"bytes": (20 if case["kl"] else 16) * n + each + 12, "flops": (12 if case["kl"] else 6) * n}
