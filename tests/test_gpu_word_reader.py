"""The reader of documents: its operators together, as a program uses them."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def corpus():
    import lda_synth
    import paper_2007_08725_amd as lda
    from paper_2007_08725_amd import word_model
    c = lda_synth.make_corpus("c1", n_docs=300)
    with lda.LDA(c.word, c.doc, c.V, c.K, c.alpha, c.beta, lda_synth.SAMPLER_SEED) as m:
        m.iterate(20)
        counts = m.counts(z=False)
    teacher = word_model.topic_teacher(counts, c.V, c.K, c.alpha, c.beta, 12)
    order = np.argsort(c.doc, kind="stable")
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(np.bincount(c.doc, minlength=c.n_docs))])).cuda()
    return c, counts, teacher, torch.from_numpy(c.word[order]).cuda(), offsets


def test_topic_teacher(corpus):
    """The most likely words of a document and their probabilities, from the tables entry by entry."""
    c, counts, (words, scores), _, _ = corpus
    assert words.shape == scores.shape == (c.n_docs, 12) and words.dtype == torch.int32
    phi = np.full((c.V, c.K), c.beta)
    for v in range(c.V):
        for i in range(counts["W_off"][v], counts["W_off"][v + 1]):
            phi[v, counts["W_topic"][i]] += counts["W_count"][i]
    phi /= np.asarray(counts["T"]) + c.V * c.beta
    for d in (0, 7, c.n_docs - 1):
        theta = np.full(c.K, c.alpha)
        for i in range(counts["D_off"][d], counts["D_off"][d + 1]):
            theta[counts["D_topic"][i]] += counts["D_count"][i]
        p = phi @ (theta / theta.sum())
        got = scores[d].double().exp().cpu().numpy()
        # sums of K products in 32 bits
        assert np.allclose(got, p[words[d].cpu().numpy()], rtol=(c.K + 8) * 4 * E, atol=0)
        assert got.min() >= np.sort(p)[-12] * (1 - 1e-5)


def batch_of(corpus, first, last):
    _, _, teacher, words, offsets = corpus
    ends = offsets[first:last + 1]
    doc = torch.repeat_interleave(torch.arange(first, last, device="cuda"), ends[1:] - ends[:-1])
    return words[ends[0]:ends[-1]], ends - ends[0], (teacher[0][doc], teacher[1][doc])


def test_gradients_follow_autograd_in_64_bits(corpus):
    """The chain of all backward passes against torch's own derivative of the same formulas."""
    from paper_2007_08725_amd.word_reader import WordReader
    c = corpus[0]
    words, offsets, teacher = batch_of(corpus, 3, 8)
    offsets = torch.cat([offsets[:2], offsets[1:]])  # an empty document among them
    rows = words.shape[0]
    model = WordReader(c.V, 40, 48, dtype=torch.float32, word_counts=np.bincount(c.word, minlength=c.V))
    dloss, dapart = torch.linspace(-1, 1, rows, device="cuda"), torch.linspace(1, 0.2, rows, device="cuda")
    loss, apart, forward = model.loss(words, offsets, teacher, 1.5)
    got = model.gradients(forward, dloss, dapart)
    p = {n: t.double().cpu().requires_grad_() for n, t in model.params.items()}
    ends, w = offsets.tolist(), words.long().cpu()
    states = []
    for a, b in zip(ends[:-1], ends[1:]):
        s = torch.zeros(40, dtype=torch.float64)
        for t in range(a, b):
            if t == a:
                e, f = torch.zeros(40, dtype=torch.float64), torch.full((40,), 0.5, dtype=torch.float64)
            else:
                e, f = p["embed"][w[t - 1]] * math.sqrt(40), torch.sigmoid(p["gate"][w[t - 1]])
            s = f * s + (1 - f) * e
            states.append(s)
    x = torch.nn.functional.layer_norm(torch.stack(states), (40,), p["norm_weight"], p["norm_bias"], 1e-5)
    a = x @ p["w_gate"].t()
    z = (a * torch.sigmoid(a) * (x @ p["w_value"].t())) @ p["weight"].t() + p["bias"]
    want = torch.logsumexp(z, 1) - z[torch.arange(rows), w]
    tw, ts = teacher[0].long().cpu(), teacher[1].double().cpu() / 1.5
    log_p = torch.log_softmax(ts, 1)
    student = torch.log_softmax(z / 1.5, 1).gather(1, tw)
    far = (log_p.exp() * (log_p - student)).sum(1)
    # sums of at most 2,000 terms in 32 bits, five deep, of the largest terms
    room = 5 * 2008 * E
    assert torch.allclose(loss.double().cpu(), want, rtol=0, atol=room * float(want.detach().abs().max()))
    assert torch.allclose(apart.double().cpu(), far, rtol=0, atol=room * float(want.detach().abs().max()))
    ((want * dloss.double().cpu()).sum() + (far * dapart.double().cpu()).sum()).backward()
    for name, t in p.items():
        scale = float(t.grad.abs().max())
        assert scale > 0 and torch.allclose(got[name].double().cpu(), t.grad, rtol=0, atol=room * scale), name


def test_a_word_at_a_time_is_the_whole(corpus):
    """Reading documents of a batch in steps gives the losses of reading them at once."""
    from paper_2007_08725_amd.word_reader import WordReader
    c = corpus[0]
    words, offsets, _ = batch_of(corpus, 0, 5)
    model = WordReader(c.V, 64, 64, dtype=torch.float32)
    whole, _, _ = model.loss(words, offsets)
    length = int((offsets[1:] - offsets[:-1]).min())
    state = model.start(5)
    for t in range(min(length, 40)):
        loss, state = model.read(state, words[offsets[:-1] + t])
        # both are within some hundred roundings of a loss of about log V
        assert torch.allclose(loss, whole[offsets[:-1] + t], rtol=0, atol=2008 * E * 10)


def test_the_same_bits_twice_and_in_every_type(corpus):
    from paper_2007_08725_amd import word_reader
    c, _, teacher, words, offsets = corpus
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        ends = []
        for _ in range(2):
            model = word_reader.WordReader(c.V, 48, 32, dtype=dtype, word_counts=np.bincount(c.word, minlength=c.V))
            losses = word_reader.train(model, words, offsets, 4, batch=1500, teacher=teacher, part=0.5)
            assert all(math.isfinite(x) for x in losses)
            ends.append(model.params)
        for n, t in ends[0].items():
            assert bool(t.isfinite().all()) and torch.equal(t, ends[1][n]), (dtype, n)


def test_the_command_runs(capsys):
    from paper_2007_08725_amd import word_model
    import json
    assert word_model.main(["--workload", "c1", "--docs", "120", "--iters", "5", "--steps", "3", "--batch", "512",
                            "--hidden", "32", "--reader", "--distil", "0.5", "--top", "8"]) == 0
    said = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    for name in ("llpt_reader", "llpt_reader_before", "llpt_word_model", "llpt_fitted_topics"):
        assert math.isfinite(said[name]) and said[name] < 0


def test_words_before():
    from paper_2007_08725_amd.word_reader import words_before
    words = torch.tensor([5, 6, 7, 8, 9], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 0, 2, 2, 5, 5], device="cuda")
    assert words_before(words, off).tolist() == [-1, 5, -1, 7, 8]
    empty = words[:0]
    assert words_before(empty, off[:1]).tolist() == []
