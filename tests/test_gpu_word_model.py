"""The word model on a fitted corpus: its pieces together, as a program uses them."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def corpus():
    import lda_synth
    import paper_2007_08725_amd as lda
    from paper_2007_08725_amd import word_model
    c = lda_synth.make_corpus("c1")
    with lda.LDA(c.word, c.doc, c.V, c.K, c.alpha, c.beta, lda_synth.SAMPLER_SEED) as m:
        m.iterate(30)
        counts = m.counts(z=False, W=False)
        fitted = m.loglik()
    proportions = word_model.topic_proportions(counts, c.K, c.alpha)
    return c, proportions, torch.from_numpy(c.word).cuda(), torch.from_numpy(c.doc).long().cuda(), fitted


def test_topic_proportions(corpus):
    c, proportions, _, _, _ = corpus
    assert proportions.shape == (c.n_docs, c.K)
    assert torch.allclose(proportions.sum(1), torch.full((c.n_docs,), float(c.K), device="cuda"), rtol=1e-5)


def test_gradients_follow_autograd_in_64_bits(corpus):
    """The chain of the three backward passes against torch's own derivative of the same formulas."""
    from paper_2007_08725_amd import word_model
    c, proportions, word, doc, _ = corpus
    model = word_model.WordModel(c.K, c.V, 48, dtype=torch.float32, word_counts=np.bincount(c.word, minlength=c.V))
    theta, words = proportions[doc[:300]], word[:300]
    weight = torch.linspace(-1, 1, 300, device="cuda")
    loss, kept = model.loss(theta, words)
    got = model.gradients(kept, weight)
    p = {n: t.double().cpu().requires_grad_() for n, t in model.params.items()}
    t = theta.double().cpu()
    x = torch.nn.functional.layer_norm(t, (c.K,), p["norm_weight"], p["norm_bias"], 1e-5)
    a = x @ p["w_gate"].t()
    h = a * torch.sigmoid(a) * (x @ p["w_value"].t())
    z = h @ p["weight"].t() + p["bias"]
    want = torch.logsumexp(z, 1) - z[torch.arange(300), words.long().cpu()]
    # sums of at most 300 (rows) and 2,000 (words) terms in 32 bits, three deep:
    # 3 * 2,000 * 2^-24 = 4e-4 of the largest terms, which the largest value bounds
    assert torch.allclose(loss.double().cpu(), want, rtol=0, atol=4e-4 * float(want.detach().abs().max()))
    (want * weight.double().cpu()).sum().backward()
    for name, tensor in p.items():
        scale = float(tensor.grad.abs().max())
        assert torch.allclose(got[name].double().cpu(), tensor.grad, rtol=0, atol=4e-4 * scale), name


def test_training_learns_more_than_the_word_frequencies(corpus):
    """Starting from the words' frequencies, training on the fitted topics gains likelihood; twice the same."""
    from paper_2007_08725_amd import word_model
    c, proportions, word, doc, fitted = corpus
    freq = np.bincount(c.word, minlength=c.V)
    ends = []
    for _ in range(2):
        model = word_model.WordModel(c.K, c.V, 64, word_counts=freq)
        before = model.llpt(proportions, word, doc)
        p = freq[freq > 0] / freq.sum()
        assert before == pytest.approx(float((p * np.log2(p)).sum()), abs=0.15)  # about the unigram entropy
        losses = word_model.train(model, proportions, word, doc, 150, batch=2048)
        assert all(math.isfinite(x) for x in losses)
        ends.append(model.llpt(proportions, word, doc))
    assert ends[0] > before + 0.3
    assert ends[0] == ends[1]
    assert math.isfinite(fitted)
