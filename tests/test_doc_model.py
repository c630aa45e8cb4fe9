"""The document model: its split on the CPU, its gradients and its training on the GPU."""
import numpy as np
import pytest


def test_hold_out_parts_the_tokens_of_each_document():
    from paper_1803_04631_amd.doc_model import hold_out
    doc_ptr = np.array([0, 5, 5, 40, 41], dtype=np.int64)
    words = np.arange(41, dtype=np.int32)
    (ptr, kept), (held_ptr, held) = hold_out(doc_ptr, words, 0.3, 7)
    assert ptr[0] == held_ptr[0] == 0 and ptr[-1] == len(kept) and held_ptr[-1] == len(held) and len(kept) + len(held) == 41
    for d in range(4):
        mine = words[doc_ptr[d]:doc_ptr[d + 1]]
        a, b = kept[ptr[d]:ptr[d + 1]], held[held_ptr[d]:held_ptr[d + 1]]
        assert np.array_equal(np.sort(np.concatenate([a, b])), mine) and np.all(np.diff(a) > 0) and np.all(np.diff(b) > 0)
    assert 5 < len(held) < 20
    again = hold_out(doc_ptr, words, 0.3, 7)
    assert np.array_equal(again[0][1], kept) and np.array_equal(again[1][0], held_ptr)
    (ptr, kept), (held_ptr, held) = hold_out(doc_ptr, words, 0.0, 7)
    assert np.array_equal(ptr, doc_ptr) and len(held) == 0 and not held_ptr.any()


@pytest.mark.gpu
def test_gradients_are_those_of_the_mean_log_probability():
    import torch
    from paper_1803_04631_amd.doc_model import DocModel, Documents, features
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, K, V = 40, 33, 701
    row_ptr = np.arange(rows + 1) * 3
    topics = np.stack([np.random.default_rng(d).choice(K, 3, replace=False) for d in range(rows)]).astype(np.uint16).reshape(-1)
    x = features(row_ptr, topics, np.arange(3 * rows, dtype=np.int32) % 7 + 1, K, 0.5)
    dense = np.full((rows, K), 0.5)
    for d in range(rows):
        dense[d, topics[3 * d:3 * d + 3]] += np.arange(3 * d, 3 * d + 3) % 7 + 1
    # (a sum, a quotient and a logarithm in fp32)
    assert np.allclose(x.cpu().numpy(), np.log(dense / dense.sum(1, keepdims=True)), rtol=0, atol=2e-6)
    model = DocModel(K, np.arange(V))
    model.weight += 0.1 * torch.randn(V, K, generator=g, device="cuda")
    model.scale += 0.1 * torch.randn(K, generator=g, device="cuda")
    lengths = torch.randint(0, 30, (rows,), generator=g, device="cuda")
    ptr = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    words = Documents(ptr, torch.randint(V, (int(ptr[-1]),), generator=g, device="cuda", dtype=torch.int32))
    logprob, grads = model.gradients(x, words)
    params = [p.double().requires_grad_() for p in (model.weight, model.bias, model.scale, model.shift)]
    y = torch.nn.functional.layer_norm(x.double(), (K,), params[2], params[3], 1e-5)
    logp = torch.log_softmax(y @ params[0].t() + params[1], 1)
    row = torch.repeat_interleave(torch.arange(rows, device="cuda"), lengths)
    want = logp[row, words.tokens.long()].mean()
    # fp32 products over 33 to 701 terms: 701 units of roundoff of the sum of magnitudes at the most, about 1e-4 of the largest entry
    assert abs(float(logprob) - want.item()) <= 1e-4 * abs(want.item())
    for got, exact in zip(grads, torch.autograd.grad(-want, params)):
        assert (got.double() - exact).abs().max() <= 1e-4 * exact.abs().max()


@pytest.mark.gpu
def test_training_raises_the_held_out_log_probability(capsys):
    import corpus_synth
    from paper_1803_04631_amd import doc_model
    c = corpus_synth.tiny(D=600, V=500, K=12, mean_len=80, seed=9)
    model, x, held, rows = doc_model.train(c.doc_ptr, c.word_ids, 500, 12, iters=60, epochs=6, batch=128)
    assert len(rows) == 7 and x.shape == (600, 12)
    # the words' frequencies alone, then ever more of the documents
    assert rows[-1][2] > rows[0][2] + 0.05 and rows[-1][1] > rows[1][1]
    again = doc_model.train(c.doc_ptr, c.word_ids, 500, 12, iters=60, epochs=2, batch=128)[3]
    assert abs(again[2][2] - rows[2][2]) <= 1e-3
    assert "epoch trained held_out norm" in capsys.readouterr().out
    top = model.score(x[:5], held.batch(0, 5, held.row_ptr[:6].tolist()), alternatives=10)
    assert top.top_ids.shape == (5, 10) and (top.entropy > 0).all() and (top.top_logprobs[:, :-1] >= top.top_logprobs[:, 1:]).all()


@pytest.mark.gpu
def test_command(tmp_path, capsys):
    import corpus_synth
    from paper_1803_04631_amd import bow, doc_model
    c = corpus_synth.tiny(D=60, V=90, K=4, mean_len=30, seed=2)
    path = tmp_path / "docword.small.txt"
    bow.save_docword(path, c.doc_ptr, c.word_ids, 90)
    doc_model.main([str(path), "--topics", "4", "--iters", "5", "--epochs", "2", "--batch", "25", "--show", "2"])
    out = capsys.readouterr().out
    assert out.count("\n") == 6 and "document 2: entropy" in out
