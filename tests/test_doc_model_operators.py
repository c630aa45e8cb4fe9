"""The document model with dropout, the policy loss and 4-bit weights: runs of these operators together."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def made(rows=40, K=33, V=701, seed=3, **how):
    from paper_1803_04631_amd.doc_model import DocModel, Documents
    g = torch.Generator(device="cuda").manual_seed(seed)
    model = DocModel(K, np.arange(V), **how)
    model.weight += 0.1 * torch.randn(V, K, generator=g, device="cuda")
    model.scale += 0.1 * torch.randn(K, generator=g, device="cuda")
    lengths = torch.randint(0, 30, (rows,), generator=g, device="cuda")
    ptr = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    words = Documents(ptr, torch.randint(V, (int(ptr[-1]),), generator=g, device="cuda", dtype=torch.int32))
    row = torch.repeat_interleave(torch.arange(rows, device="cuda"), lengths)
    return model, torch.randn(rows, K, generator=g, device="cuda"), words, row, g


def logp64(model, x, mask=None):
    params = [p.double().requires_grad_() for p in (model.weight, model.bias, model.scale, model.shift)]
    y = torch.nn.functional.layer_norm(x.double(), x.shape[1:], params[2], params[3], 1e-5)
    if mask is not None:
        y = y * mask
    return params, torch.log_softmax(y @ params[0].t() + params[1], 1)


def same_gradients(grads, loss, params):
    # fp32 products over up to 701 terms: about 1e-4 of the largest entry at the most
    for got, exact in zip(grads, torch.autograd.grad(loss, params)):
        assert (got.double() - exact).abs().max() <= 1e-4 * exact.abs().max()


def test_gradients_with_dropout():
    from paper_1803_04631_amd import operators
    model, x, words, row, _ = made(dropout=0.3, seed=3)
    for steps in (0, 5):
        model.steps = steps
        logprob, grads = model.gradients(x, words)
        kept = operators.dropout(torch.ones_like(x), 0.3, model.seed, steps)
        assert 0.5 < float((kept != 0).double().mean()) < 0.9
        params, logp = logp64(model, x, (kept != 0).double() / 0.7)
        want = logp[row, words.tokens.long()].mean()
        assert abs(float(logprob) - want.item()) <= 1e-4 * abs(want.item())
        same_gradients(grads, -want, params)
    a = model.score(x, words).logprobs                                    # scoring drops nothing
    assert (a.double() - logp64(model, x)[1][row, words.tokens.long()]).abs().max() <= 1e-4


def test_policy_gradients():
    model, x, words, row, g = made(seed=4)
    n = len(words.tokens)
    params, logp = logp64(model, x)
    l = logp[row, words.tokens.long()]
    old = (l.detach() + 0.3 * torch.randn(n, generator=g, device="cuda")).float()
    reference = (l.detach() + 0.3 * torch.randn(n, generator=g, device="cuda")).float()
    advantages = torch.randn(n, generator=g, device="cuda")
    got, grads = model.policy_gradients(x, words, old, advantages, reference=reference, low=0.2, high=0.3, kl=0.1, entropy=0.05)
    ratio, d = torch.exp(l - old.double()), reference.double() - l
    least = torch.minimum(ratio * advantages.double(), ratio.clamp(0.8, 1.3) * advantages.double())
    loss = (0.1 * (torch.exp(d) - d - 1) - least).mean()
    entropy = -(logp.exp() * logp).sum(1).mean()
    # log-probabilities of about 7 are off by 1e-6: so are ratios, of which n are averaged
    assert abs(float(got.loss) - loss.item()) <= 1e-5
    border = torch.minimum((l - old - math.log(0.8)).abs(), (l - old - math.log(1.3)).abs())
    assert border.min() > 1e-5
    same_gradients(grads, loss - 0.05 * entropy, params)


def test_policy_steps_leave_no_features_out():
    model, x, words, _, g = made(dropout=0.5, seed=4)
    whole = made(seed=4)[0]
    old, advantages = model.score(x, words).logprobs, torch.randn(len(words.tokens), generator=g, device="cuda")
    a, b = (m.policy_gradients(x, words, old, advantages) for m in (model, whole))
    assert torch.equal(a[0].grad_logprobs, b[0].grad_logprobs) and all(torch.equal(u, v) for u, v in zip(a[1], b[1]))
    assert float(a[0].clipped) == 0.0                                      # every ratio is 1
    assert not torch.equal(model.gradients(x, words)[1][0], whole.gradients(x, words)[1][0])


@pytest.mark.parametrize("max_norm", [1e-3, 1e3])
def test_a_policy_step_descends_its_gradient(max_norm):
    model, x, words, _, g = made(seed=8)
    n = len(words.tokens)
    old = model.score(x, words).logprobs + 0.1 * torch.randn(n, generator=g, device="cuda")
    advantages = torch.randn(n, generator=g, device="cuda")
    want, grads = model.policy_gradients(x, words, old, advantages, entropy=0.01)
    before = [p.clone() for p in (model.weight, model.bias, model.scale, model.shift)]
    got = model.policy_step(x, words, old, advantages, 0.25, max_norm, entropy=0.01)
    assert model.steps == 1 and all(torch.equal(u, v) for u, v in zip(got, want))
    norm = math.sqrt(sum(float(v.double().square().sum()) for v in grads))
    factor = min(1.0, max_norm / norm)
    assert (factor < 1) == (max_norm < 1)
    for p, was, grad in zip((model.weight, model.bias, model.scale, model.shift), before, grads):
        step = 0.25 * factor * grad.double()
        # a factor and a product in fp32, another product and a difference: 2^-24 of what is made, a few times
        assert (p.double() - (was.double() - step)).abs().max() <= (2.0 ** -24 * (was.abs() + 8 * step.abs())).max()
        assert float(step.abs().max()) > 0


def test_suggested_words_and_what_they_are_worth():
    """What each step is given: words of the right documents, an advantage of 1 where the document holds the word less the mean, log-probabilities of
    the model that drew them and of the model as it was at first."""
    from paper_1803_04631_amd.doc_model import suggest_words
    said, given = [], []
    for run in range(2):
        model, x, words, row, _ = made(rows=25, seed=9)
        first, step = logp64(model, x)[1].detach(), model.policy_step

        def watched(x_, w, old, advantages, rate, max_norm, reference=None, kl=0.0):
            given.append((w, old, advantages, reference, kl, logp64(model, x)[1].detach()))
            return step(x_, w, old, advantages, rate, max_norm, reference=reference, kl=kl)

        model.policy_step = watched
        said.append(suggest_words(model, x, words, rounds=3, draws=7, steps=2, rate=0.5, kl=0.03, seed=5))
    assert said[0] == said[1] and [r[0] for r in said[0]] == [1, 2, 3] and len(given) == 12
    holds = set(zip(row.tolist(), words.tokens.tolist()))
    for k, (w, old, advantages, reference, kl, logp) in enumerate(given[:6]):
        assert torch.equal(w.row_ptr, 7 * torch.arange(26, device="cuda")) and kl == 0.03
        document = torch.arange(25, device="cuda").repeat_interleave(7)
        worth = torch.tensor([(d, t) in holds for d, t in zip(document.tolist(), w.tokens.tolist())], dtype=torch.float64, device="cuda")
        assert (advantages.double() - (worth - worth.mean())).abs().max() <= 1e-6
        assert abs(said[0][k // 2][1] - float(worth.mean())) <= 1e-6
        at = document, w.tokens.long()
        assert (reference.double() - first[at]).abs().max() <= 1e-4
        if k % 2 == 0:                                                     # the model that drew them
            assert (old.double() - logp[at]).abs().max() <= 1e-4
        else:                                                              # the same words and log-probabilities, by a model that is a step further
            assert torch.equal(w.tokens, given[k - 1][0].tokens) and torch.equal(old, given[k - 1][1]) and not torch.equal(logp, given[k - 1][5])
    for _, held, kl, clipped in said[0]:
        assert 0 <= held <= 1 and 0 <= clipped <= 1 and kl > 0
    model, x, words, _, _ = made(rows=25, seed=9)
    (_, _, kl, clipped), = suggest_words(model, x, words, rounds=1, draws=7, steps=1)
    assert abs(kl) <= 1e-9 and clipped == 0                                # before the first step the model is as it was


def test_packed_scores_are_those_of_the_packed_weights():
    from paper_1803_04631_amd import operators
    model, x, words, row, _ = made(rows=100, K=70, V=1003, seed=5)
    packed = model.packed(dtype=torch.float32)
    y = operators.layer_norm(x, model.scale, model.shift)[0]
    held = operators.mx4_dequantize(operators.mx4_quantize(y)).double()
    logits = held @ operators.mx4_dequantize(packed.weight).double().t() + model.bias.double()
    want = torch.log_softmax(logits, 1)[row, words.tokens.long()]
    got = packed.score(x, words, alternatives=5)
    # sums of 70 terms of up to 3 in fp32, logits of up to 10
    assert (got.logprobs.double() - want).abs().max() <= 2e-5
    full = model.score(x, words)
    # a product of 4-bit numbers: an eighth of a feature and an eighth of a weight off, some 0.16 of logits that spread by 0.8, 100 rows of 30 words averaged
    assert abs(float((got.logprobs - full.logprobs).mean())) < 0.1
    assert got.top_ids.shape == (100, 5) and (got.entropy > 0).all()
    model.weight.zero_()                                                   # (the packed model is as it was)
    assert torch.equal(packed.score(x, words).logprobs, got.logprobs)


def test_logits_of_packed_weights_are_rounded_once_more():
    """The scores of a packed model are those of its fp32 logits, each rounded to bf16."""
    from paper_1803_04631_amd import operators
    model, x, words, row, _ = made(rows=100, K=70, V=1003, seed=5)
    fine, coarse = model.packed(torch.float32), model.packed()
    assert fine.dtype == torch.float32 and coarse.dtype == torch.bfloat16 and torch.equal(fine.weight.codes, coarse.weight.codes)
    y = operators.layer_norm(x, model.scale, model.shift)[0]
    logits = operators.mx4_linear(y, fine.weight, fine.bias)
    assert torch.equal(operators.mx4_linear(y, coarse.weight, coarse.bias, dtype=torch.bfloat16), logits.bfloat16())
    at = row, words.tokens.long()
    want = torch.log_softmax(logits.bfloat16().double(), 1)[at]
    assert (coarse.score(x, words).logprobs.double() - want).abs().max() <= 2e-5
    # a logit is off by 2^-8 of itself at the most, and so is the logarithm of the sum
    off = 2.0 ** -8 * (logits[at].abs() + logits.abs().amax(1)[row])
    assert ((coarse.score(x, words).logprobs - fine.score(x, words).logprobs).abs() <= off + 1e-4).all()


def test_a_step_in_a_graph_draws_new_masks():
    """Forward, loss and backward of a step captured once: each replay has the mask of the step's number that it finds on the GPU."""
    from paper_1803_04631_amd import operators
    model, x, words, row, _ = made(seed=6)
    weights = torch.full((len(words.tokens),), -1.0 / len(words.tokens), device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def gradient(step):
        y, mean, rstd = operators.layer_norm(x, model.scale, model.shift)
        operators.dropout(y, 0.4, 9, step, out=y)
        logits = torch.addmm(model.bias, y, model.weight.t())
        grad = operators.token_logprobs_grad(logits, words.tokens, weights, words.row_ptr, out=logits)[1]
        grad_y = operators.dropout_backward(grad @ model.weight, 0.4, 9, step)
        return operators.layer_norm_backward(grad_y, x, mean, rstd, model.scale)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        gradient(step)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gradient(step)
        step += 1
    seen = []
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = gradient(k)
        # (the library products of a captured stream may be others: 701 terms in fp32)
        assert all((a - b).abs().max() <= 1e-4 * b.abs().max() for a, b in zip(out, want))
        seen.append(out[0].clone())
    assert all(not torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])


def test_training_with_dropout_suggestions_and_packed_weights(tmp_path, capsys):
    import corpus_synth
    from paper_1803_04631_amd import bow, doc_model
    c = corpus_synth.tiny(D=80, V=90, K=4, mean_len=40, seed=2)
    path = tmp_path / "docword.small.txt"
    bow.save_docword(path, c.doc_ptr, c.word_ids, 90)
    doc_model.main([str(path), "--topics", "4", "--iters", "5", "--epochs", "2", "--batch", "30", "--show", "2", "--dropout", "0.2", "--suggest", "2", "--packed"])
    out = capsys.readouterr().out
    assert "round held kl clipped" in out and "in 4 bits" in out and "document 2: entropy" in out
    a = doc_model.train(c.doc_ptr, c.word_ids, 90, 4, iters=5, epochs=2, batch=30, dropout=0.2)
    b = doc_model.train(c.doc_ptr, c.word_ids, 90, 4, iters=5, epochs=2, batch=30, dropout=0.2)
    assert abs(a[3][-1][2] - b[3][-1][2]) <= 1e-4 and a[0].steps == b[0].steps == 6        # the same masks in both runs


def test_what_is_held_out_is_not_rewarded(tmp_path, capsys, monkeypatch):
    """The command rewards words of the tokens that it sampled, and its last figures are of tokens that no step has seen."""
    import corpus_synth
    from paper_1803_04631_amd import bow, doc_model
    c = corpus_synth.tiny(D=80, V=90, K=4, mean_len=40, seed=2)
    path = tmp_path / "docword.small.txt"
    bow.save_docword(path, c.doc_ptr, c.word_ids, 90)
    doc_ptr, word_ids, _ = bow.load_docword(str(path))
    (ptr, words), (held_ptr, held_words) = doc_model.hold_out(doc_ptr, word_ids, 0.2, 4631)
    given, suggest = [], doc_model.suggest_words

    def watched(model, x, documents, *args, **how):
        given.append((model, x, documents))
        return suggest(model, x, documents, *args, **how)

    monkeypatch.setattr(doc_model, "suggest_words", watched)
    doc_model.main([str(path), "--topics", "4", "--iters", "5", "--epochs", "1", "--batch", "30", "--suggest", "2", "--packed"])
    model, x, documents = given[0]
    assert len(given) == 1 and len(x) == 30
    assert np.array_equal(documents.row_ptr.cpu().numpy(), ptr[:31]) and np.array_equal(documents.tokens.cpu().numpy(), words[:ptr[30]])
    trained = doc_model.train_documents(doc_ptr, word_ids, 90, 4, iters=5, epochs=1, batch=30)
    assert np.array_equal(trained.held.tokens.cpu().numpy(), held_words) and np.array_equal(trained.held.row_ptr.cpu().numpy(), held_ptr)
    assert np.array_equal(trained.seen.tokens.cpu().numpy(), words) and torch.equal(trained.features[:30], x)
    held = model.score(trained.features, trained.held).logprobs.double().mean()
    said = capsys.readouterr().out.split("held_out in 32 bits ")[1].split(",")[0]
    assert abs(float(said) - float(held)) <= 1e-4                          # four places; scores in other batches
