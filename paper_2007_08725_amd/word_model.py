"""A neural word model on a fitted corpus: p(word | topics of its document).

The sampler fits topics; this model predicts words from them.  A token's input
is its document's topic proportions (D[d][k] + alpha) / (len(d) + K alpha), which
go through a layer norm, a gated layer and a softmax over the vocabulary:

    x = layer_norm(K * theta_d);  h = act(x w_gate^T) * (x w_value^T)
    p(v) = softmax(h weight^T + bias)_v

trained on the corpus' tokens with Adam.  Its score is the log-likelihood per
token in base 2, as ``LDA.loglik`` gives it for the fitted counts, so the two
stand side by side.  Scoring new words of a document needs no sampling.

With ``--reader`` a second model is trained, that needs no topics of a document
but reads its words in order (``word_reader.py``), from the words alone or, with
``--distil``, from the fitted topics' most likely words for each document too.
Like the others it is scored on the documents that it was trained on, whose words
it may know by heart: that says nothing of new ones.

    python -m paper_2007_08725_amd.word_model --workload c1 --iters 50 --steps 300 --reader --distil 0.5
"""
import argparse
import json
import math
import sys
import time

import numpy as np
import torch

from . import ops


def topic_proportions(counts, K: int, alpha: float, device="cuda"):
    """K times the topic proportions of every document, [M, K] in float32, from ``LDA.counts`` (1 on average)."""
    off = np.asarray(counts["D_off"])
    length = np.diff(off)
    rows = torch.from_numpy(np.repeat(np.arange(length.size), length)).to(device)
    theta = torch.full((length.size, K), float(alpha), device=device)
    entries = torch.from_numpy(np.asarray(counts["D_topic"], np.int64)).to(device)
    theta[rows, entries] += torch.from_numpy(np.asarray(counts["D_count"], np.float32)).to(device)
    return theta * (K / theta.sum(1, keepdim=True))


def topic_teacher(counts, V: int, K: int, alpha: float, beta: float, top: int = 32, device="cuda"):
    """The fitted topics' most likely words of every document and their log-probabilities: int32 and float32 [M, top].

    p(v | d) = sum_k theta_dk phi_kv with theta as ``topic_proportions`` and phi_kv = (W[v][k] + beta) / (T[k] + V beta).
    """
    off, total = np.asarray(counts["W_off"]), np.asarray(counts["T"], np.float64)
    rows = torch.from_numpy(np.repeat(np.arange(V), np.diff(off))).to(device)
    phi = torch.full((V, K), float(beta), device=device)
    entries = torch.from_numpy(np.asarray(counts["W_topic"], np.int64)).to(device)
    phi[rows, entries] += torch.from_numpy(np.asarray(counts["W_count"], np.float32)).to(device)
    phi /= torch.from_numpy(total + V * beta).to(device=device, dtype=torch.float32)
    theta = topic_proportions(counts, K, alpha, device) / K
    words, scores = [], []
    for i in range(0, theta.shape[0], 1024):
        p, v = torch.topk(theta[i:i + 1024] @ phi.t(), top)
        words.append(v.to(torch.int32))
        scores.append(torch.log(p))
    return torch.cat(words), torch.cat(scores)


class Trained:
    """Parameters in float32 under ``params``, their Adam averages, and the type that products run in."""

    def _start(self, params, dtype):
        self.params, self.dtype = params, dtype
        # half precision takes the gradients of this many times the mean loss: those of the mean over a batch of
        # thousands are below its normal numbers
        self._loss_scale = 1024.0 if dtype == torch.float16 else 1.0
        self._moments = {n: (torch.zeros_like(p), torch.zeros_like(p)) for n, p in params.items()}
        self._steps = 0

    def _cast(self):
        # the softmax's bias stays in float32
        return {n: p if n == "bias" else p.to(self.dtype) for n, p in self.params.items()}

    def _adam(self, grads, lr: float):
        """One Adam step with gradients of ``_loss_scale`` times the loss."""
        self._steps += 1
        c1, c2 = 1 - 0.9 ** self._steps, 1 - 0.999 ** self._steps
        for name, param in self.params.items():
            g = grads[name].float()
            if self._loss_scale != 1.0:
                g = g / self._loss_scale
            m, v = self._moments[name]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.999).addcmul_(g, g, value=0.001)
            param.addcdiv_(m / c1, (v / c2).sqrt_().add_(1e-8), value=-lr)


def word_bias(word_counts, V: int, device):
    """The logarithm of the words' frequencies, from which the softmax's bias starts."""
    freq = torch.ones(V, device=device) if word_counts is None else torch.as_tensor(
        np.asarray(word_counts), device=device).float() + 0.5
    return torch.log(freq / freq.sum())


class WordModel(Trained):
    """The model's parameters (float32) and their training; products run in ``dtype``."""

    def __init__(self, K: int, V: int, hidden: int = 256, act: str = "silu", dtype=torch.bfloat16, word_counts=None,
                 seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(*shape, generator=gen, device=device) * scale

        self.act = act
        self._start(dict(norm_weight=torch.ones(K, device=device), norm_bias=torch.zeros(K, device=device),
                         w_gate=normal(hidden, K, scale=K ** -0.5), w_value=normal(hidden, K, scale=K ** -0.5),
                         weight=normal(V, hidden, scale=0.1 * hidden ** -0.5),
                         bias=word_bias(word_counts, V, device)), dtype)

    def loss(self, theta, words):
        """Negative log-likelihood of each word (natural log), and what the backward pass takes."""
        p = self._cast()
        theta = theta.to(self.dtype)
        x, mean, rstd = ops.layer_norm(theta, p["norm_weight"], p["norm_bias"])
        h = ops.gated(x, p["w_gate"], p["w_value"], self.act)
        loss, lse = ops.softmax_xent(h, p["weight"], words, p["bias"])
        return loss, (p, theta, mean, rstd, x, h, lse, words)

    def gradients(self, kept, dloss):
        """Gradients of sum(dloss * loss) by the parameters' names."""
        p, theta, mean, rstd, x, h, lse, words = kept
        dh, dweight, dbias = ops.softmax_xent_backward(dloss, lse, h, p["weight"], words, p["bias"])
        dx, dw_gate, dw_value = ops.gated_backward(dh, x, p["w_gate"], p["w_value"], self.act)
        _, dnorm_weight, dnorm_bias = ops.layer_norm_backward(dx, theta, p["norm_weight"], mean, rstd)
        return dict(norm_weight=dnorm_weight, norm_bias=dnorm_bias, w_gate=dw_gate, w_value=dw_value, weight=dweight,
                    bias=dbias)

    def step(self, theta, words, lr: float = 1e-2):
        """One Adam step on a batch of tokens; returns the batch's mean loss, on the device."""
        loss, kept = self.loss(theta, words)
        grads = self.gradients(kept, torch.full_like(loss, self._loss_scale / loss.shape[0]))
        self._adam(grads, lr)
        return loss.mean()

    def llpt(self, proportions, word, doc, batch: int = 8192):
        """Log-likelihood per token, log base 2."""
        total = torch.zeros((), dtype=torch.float64, device=proportions.device)
        for i in range(0, word.shape[0], batch):
            loss, _ = self.loss(proportions[doc[i:i + batch]], word[i:i + batch])
            total -= loss.double().sum()
        return float(total) / (word.shape[0] * math.log(2))


def train(model, proportions, word, doc, steps: int, batch: int = 4096, lr: float = 1e-2, seed: int = 1):
    """``steps`` Adam steps on random tokens (``word`` and ``doc`` on the device); returns the losses."""
    gen = torch.Generator(device=word.device).manual_seed(seed)
    losses = []
    for _ in range(steps):
        pick = torch.randint(0, word.shape[0], (batch,), generator=gen, device=word.device)
        losses.append(model.step(proportions[doc[pick]], word[pick], lr))
    return [float(x) for x in losses]


def _check(ap, args):
    """Refuses what the reader cannot be trained with, before anything is fitted, and fills in what was not given."""
    if not 0.0 <= args.distil <= 1.0:
        ap.error("--distil must be 0 to 1")
    if args.distil > 0 and not args.reader:
        ap.error("--distil needs --reader")
    for name, default in (("top", 32), ("temperature", 1.0)):
        if getattr(args, name) is None:
            setattr(args, name, default)
        elif not args.distil > 0:
            ap.error("--%s needs --distil" % name)
    if not 1 <= args.top <= ops.MAX_TOP:
        ap.error("--top must be 1 to %d" % ops.MAX_TOP)
    most = float(np.finfo(np.float32).max)  # the operator takes it in single precision
    if not 1.0 / most < args.temperature < most:
        ap.error("--temperature and its reciprocal must be finite and positive")


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="c1", choices=["c1", "c2"])
    ap.add_argument("--docs", type=int, default=0, help="documents of the corpus (0 = all)")
    ap.add_argument("--iters", type=int, default=50, help="iterations of the sampler")
    ap.add_argument("--steps", type=int, default=300, help="training steps of the word model")
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--reader", action="store_true",
                    help="train a reader of the words in order too (scored on the documents that it was trained on)")
    ap.add_argument("--distil", type=float, default=0.0, help="the fitted topics' part of the reader's loss, 0 to 1")
    ap.add_argument("--top", type=int, help="words that the fitted topics list for a document (32)")
    ap.add_argument("--temperature", type=float, help="of the fitted topics' and the reader's probabilities (1)")
    ap.add_argument("--eval-tokens", type=int, default=1 << 20, help="tokens scored at the end, from the corpus' start")
    args = ap.parse_args(argv)
    _check(ap, args)

    import lda_synth

    from . import LDA

    torch.cuda.set_device(0)
    c = lda_synth.make_corpus(args.workload, **(dict(n_docs=args.docs) if args.docs else {}))
    with LDA(c.word, c.doc, c.V, c.K, c.alpha, c.beta, lda_synth.SAMPLER_SEED) as m:
        m.iterate(args.iters)
        fitted = m.loglik()
        counts = m.counts(z=False, W=args.reader)
    proportions = topic_proportions(counts, c.K, c.alpha)
    word = torch.from_numpy(c.word).cuda()
    doc = torch.from_numpy(c.doc).long().cuda()
    freq = np.bincount(c.word, minlength=c.V)
    model = WordModel(c.K, c.V, args.hidden, word_counts=freq)
    some = slice(0, min(args.eval_tokens, c.N))
    before = model.llpt(proportions, word[some], doc[some])
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    losses = train(model, proportions, word, doc, args.steps, args.batch, args.lr)
    elapsed = time.perf_counter() - t0
    said = dict(workload=args.workload, tokens=c.N, V=c.V, K=c.K, llpt_fitted_topics=fitted,
                llpt_word_model_before=before, llpt_word_model=model.llpt(proportions, word[some], doc[some]),
                first_loss=losses[0] if losses else None, last_loss=losses[-1] if losses else None,
                ms_per_step=elapsed * 1e3 / max(1, args.steps))
    if args.reader:
        from . import word_reader
        said.update(word_reader.fit(c, args, freq, topic_teacher(counts, c.V, c.K, c.alpha, c.beta, args.top)
                                    if args.distil > 0 else None))
    print(json.dumps(said))
    return 0


if __name__ == "__main__":
    sys.exit(main())
