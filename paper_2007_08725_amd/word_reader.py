"""A model that reads a document's words in order: p(word | the words before it).

It needs no topics of the document, so that a new one is scored by reading it
once, or a word at a time.  Each word has two rows in the model, what it adds to
the state of the document and how much of the state it lets stay:

    e_t = sqrt(width) * embed[word_{t-1}], g_t = gate[word_{t-1}]
    s_t = f s_{t-1} + (1 - f) e_t,  f = sigmoid(g_t)       (anew in each document)
    h = act(norm(s_t) w_gate^T) * (norm(s_t) w_value^T)
    p(v) = softmax(h weight^T + bias)_v

The first word of a document is read from a state of zeros (the word before it
is none: -1).  It is trained on the words that come next, and on a teacher's
most likely words of each document (``word_model.topic_teacher``) beside them.
"""
import math
import time

import numpy as np
import torch

from . import ops
from .word_model import Trained, word_bias


def words_before(words, offsets):
    """Each word's predecessor in its document, -1 for the first ones (int32; ``offsets`` as ``LDA.counts`` has D_off's)."""
    before = torch.cat([words.new_full((1,), -1), words[:-1]])[:words.shape[0]]
    first = offsets[:-1][offsets[1:] > offsets[:-1]]
    before[first] = -1
    return before


class WordReader(Trained):
    """The reader's parameters (float32) and their training; products run in ``dtype``."""

    def __init__(self, V: int, width: int = 256, hidden: int = 256, act: str = "silu", dtype=torch.bfloat16,
                 word_counts=None, seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(*shape, generator=gen, device=device) * scale

        self.V, self.width, self.act = V, width, act
        # gates start between a memory of a few words and one of a hundred
        keep = torch.linspace(1.0, 5.0, width, device=device)
        self._start(dict(embed=normal(V, width, scale=width ** -0.5), gate=normal(V, width, scale=0.1) + keep,
                         norm_weight=torch.ones(width, device=device), norm_bias=torch.zeros(width, device=device),
                         w_gate=normal(hidden, width, scale=width ** -0.5),
                         w_value=normal(hidden, width, scale=width ** -0.5),
                         weight=normal(V, hidden, scale=0.1 * hidden ** -0.5),
                         bias=word_bias(word_counts, V, device)), dtype)

    def _hidden(self, p, s):
        x, mean, rstd = ops.layer_norm(s, p["norm_weight"], p["norm_bias"])
        return x, mean, rstd, ops.gated(x, p["w_gate"], p["w_value"], self.act)

    def loss(self, words, offsets, teacher=None, temperature: float = 1.0):
        """Negative log-likelihood of each word (natural log), the distance from ``teacher`` (its words and scores, a
        row for each word) or None, and what the backward pass takes."""
        p = self._cast()
        before = words_before(words, offsets)
        e = ops.embedding(before, p["embed"], math.sqrt(self.width))
        g = ops.embedding(before, p["gate"])
        s, _, kept = ops.recurrence(e, g, offsets)
        x, mean, rstd, h = self._hidden(p, s)
        loss, lse = ops.softmax_xent(h, p["weight"], words, p["bias"])
        apart = taught = None
        if teacher is not None:
            given = (h, p["weight"], *teacher, p["bias"], temperature)
            apart, *taught = ops.softmax_distill(*given)
            taught = (*taught, *given)
        return loss, apart, (p, words, offsets, before, e, g, s, kept, x, mean, rstd, h, lse, taught)

    def gradients(self, forward, dloss, dapart=None):
        """Gradients of sum(dloss * loss) + sum(dapart * apart) by the parameters' names."""
        p, words, offsets, before, e, g, s, kept, x, mean, rstd, h, lse, taught = forward
        dh, dweight, dbias = ops.softmax_xent_backward(dloss, lse, h, p["weight"], words, p["bias"])
        if taught is not None:
            more = ops.softmax_distill_backward(dapart, *taught)
            # the weight's in 32 bits, as the step takes it: no third rounding to the products' type
            dh, dweight, dbias = dh + more[0], dweight.float() + more[1], dbias + more[2]
        dx, dw_gate, dw_value = ops.gated_backward(dh, x, p["w_gate"], p["w_value"], self.act)
        ds, dnorm_weight, dnorm_bias = ops.layer_norm_backward(dx, s, p["norm_weight"], mean, rstd)
        de, dg, _ = ops.recurrence_backward(ds, e, g, offsets, kept)
        return dict(embed=ops.embedding_backward(de, before, self.V, math.sqrt(self.width)),
                    gate=ops.embedding_backward(dg, before, self.V), norm_weight=dnorm_weight, norm_bias=dnorm_bias,
                    w_gate=dw_gate, w_value=dw_value, weight=dweight, bias=dbias)

    def step(self, words, offsets, teacher=None, part: float = 0.5, temperature: float = 1.0, lr: float = 1e-2):
        """One Adam step on whole documents; returns the mean loss of the words, on the device.

        With a ``teacher`` its distance is ``part`` of what is minimised.
        """
        loss, apart, forward = self.loss(words, offsets, teacher, temperature)
        each = torch.full_like(loss, self._loss_scale / loss.shape[0])
        grads = self.gradients(forward, each if apart is None else (1 - part) * each,
                               None if apart is None else part * each)
        self._adam(grads, lr)
        return loss.mean()

    def llpt(self, words, offsets, batch: int = 65536):
        """Log-likelihood per token, log base 2, of whole documents."""
        ends = offsets.tolist()
        total, first = torch.zeros((), dtype=torch.float64, device=words.device), 0
        while first < len(ends) - 1:
            last = first + 1  # as many documents as a batch holds, one at least
            while last < len(ends) - 1 and ends[last + 1] - ends[first] <= batch:
                last += 1
            part = words[ends[first]:ends[last]]
            if part.shape[0]:
                loss, _, _ = self.loss(part, offsets[first:last + 1] - ends[first])
                total -= loss.double().sum()
            first = last
        return float(total) / (max(1, ends[-1] - ends[0]) * math.log(2))

    def start(self, docs: int):
        """The state of ``docs`` documents of which nothing is read, for the parameters as they are now."""
        device = self.params["bias"].device
        return (self._cast(), torch.zeros(docs, self.width, dtype=self.dtype, device=device),
                torch.zeros(docs, self.width, device=device))

    def read(self, state, words):
        """Scores the next word of each document and reads it: ``(loss, state)``, as ``loss`` has them for the whole.

        A document that has ended among others has the word -1: its loss is 0, and what its state is then says nothing.
        """
        p, s, exact = state
        _, _, _, h = self._hidden(p, s)
        loss, _ = ops.softmax_xent(h, p["weight"], words, p["bias"])
        e = ops.embedding(words, p["embed"], math.sqrt(self.width))
        g = ops.embedding(words, p["gate"])
        return loss, (p, *ops.recurrence_step(e, g, exact))


def train(model, words, offsets, steps: int, batch: int = 4096, lr: float = 1e-2, teacher=None, part: float = 0.5,
          temperature: float = 1.0, seed: int = 1):
    """``steps`` Adam steps on some ``batch`` words of random whole documents (``teacher``: words and scores by
    document); returns the losses."""
    gen = np.random.default_rng(seed)
    ends = offsets.cpu().numpy()
    length = np.diff(ends)
    full = np.nonzero(length)[0]
    losses = []
    for _ in range(steps):
        many = max(1, min(full.size, round(batch / length[full].mean())))
        docs = gen.choice(full, many, replace=False)
        at = np.concatenate([np.arange(ends[d], ends[d + 1]) for d in docs])
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(length[docs])])).to(offsets.device)
        given = None
        if teacher is not None:
            rows = torch.from_numpy(np.repeat(docs, length[docs])).to(offsets.device)
            given = teacher[0][rows], teacher[1][rows]
        losses.append(model.step(words[torch.from_numpy(at).to(words.device)], off, given, part, temperature, lr))
    return [float(x) for x in losses]


def fit(corpus, args, word_counts, teacher=None):
    """The reader of the ``word_model`` command: trained and scored on the corpus' documents."""
    order = np.argsort(corpus.doc, kind="stable")
    words = torch.from_numpy(corpus.word[order]).cuda()
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(np.bincount(corpus.doc, minlength=corpus.n_docs))])
                               .astype(np.int64)).cuda()
    some = int(torch.searchsorted(offsets, min(args.eval_tokens, corpus.N)))
    model = WordReader(corpus.V, args.hidden, args.hidden, word_counts=word_counts)
    before = model.llpt(words, offsets[:some + 1])
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    losses = train(model, words, offsets, args.steps, args.batch, args.lr, teacher, args.distil, args.temperature)
    elapsed = time.perf_counter() - t0
    return dict(llpt_reader_before=before, llpt_reader=model.llpt(words, offsets[:some + 1]),
                llpt_reader_of="documents that it was trained on",
                reader_first_loss=losses[0] if losses else None, reader_last_loss=losses[-1] if losses else None,
                reader_ms_per_step=elapsed * 1e3 / max(1, args.steps))
