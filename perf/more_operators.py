"""Measured cases of the operators for word models that read a document's words
in order: word embedding, gated linear recurrence, and distillation from a
teacher's top words, forward and with their gradients.

The reader of a document embeds its words, runs a gated state over them that
starts anew with each document, and scores the vocabulary; it is trained on the
next word and on what another model (the fitted topics) gives its most likely
words.  A case is one operator on one shape:

  pass = "forward"  serving or scoring: the operator's outputs alone
  pass = "train"    forward, then the backward pass for given gradients
  pass = "step"     (recurrence) one more word for each of a batch of documents

Vocabularies are those of this repository's corpora (2,000, 102,000, 141,000),
lengths of documents their means (about 92 and 332 words), widths its topic
counts (16, 1,000), hidden widths of powers of two and odd sizes between.
Where ``own`` is false the operators are computed in their plain form
(elementary torch operations in 32 bits), else by the library's kernels.
``exact`` gives the definitions in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _embed(name, dtype, way, rows, width, vocab):
    return _named(name, dict(op="embed", dtype=dtype, way=way, rows=rows, width=width, vocab=vocab))


def _recur(name, dtype, way, rows, width, docs, joint, state):
    return _named(name, dict(op="recur", dtype=dtype, way=way, rows=rows, width=width, docs=docs, joint=joint,
                             state=state))


def _distill(name, dtype, way, rows, width, vocab, top, bias, temperature):
    return _named(name, dict(op="distill", dtype=dtype, way=way, rows=rows, width=width, vocab=vocab, top=top,
                             bias=bias, temperature=temperature))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one word looked up while a document is served: latency alone
        _embed("embed_one_word", "bf16", "forward", 1, 1024, 141000),
        # a training batch of words of the largest vocabulary: most of the gradient's rows are zero
        _embed("embed_batch", "bf16", "train", 65536, 1024, 141000),
        # all of a small corpus in single precision, odd width: few words, each many times
        _embed("embed_small_corpus_f32", "f32", "train", 50000, 257, 2000),
        # a million words of a news-sized corpus in half precision: the most frequent one is a tenth of them
        _embed("embed_news_f16", "f16", "train", 1 << 20, 512, 102000),
        # the next word of one document in serving
        _recur("recur_next_word", "bf16", "step", 1, 1024, 1, False, True),
        # a training batch of whole documents of some 332 words; values and gates are halves of one matrix
        _recur("recur_documents", "bf16", "train", 65536, 1024, 197, True, False),
        # one long document, continued from a state, odd width, single precision
        _recur("recur_one_long_f32", "f32", "train", 65537, 257, 1, False, True),
        # scoring many short documents of some 92 words by their topics in half precision
        _recur("recur_score_f16", "f16", "forward", 262144, 1000, 2849, False, False),
        # one position's distance from its teacher, against the largest vocabulary
        _distill("distill_one_word", "bf16", "forward", 1, 1024, 141000, 32, True, 1.0),
        # a training batch against the largest vocabulary
        _distill("distill_batch", "bf16", "train", 8192, 1024, 141000, 32, True, 1.0),
        # a small corpus in single precision, every size ragged, softened
        _distill("distill_small_f32", "f32", "train", 413, 257, 2000, 20, False, 2.0),
        # a training batch of a news-sized vocabulary in half precision, a longer list, softened
        _distill("distill_news_f16", "f16", "train", 4096, 512, 102000, 64, False, 1.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of [lo, hi], even over the logarithm; half of them multiples of 8, the others as they fall."""
    n = _log_int(rng, lo, hi)
    if n > 16 and rng.random() < 0.5:
        n = min(hi // 8 * 8, (n + 7) // 8 * 8)
    return max(lo, n)


def draw(rng):
    op = rng.choice(["embed", "embed", "recur", "recur", "recur", "distill", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    way = rng.choice(["forward", "train", "train"])
    if op == "embed":
        while True:
            rows, width, vocab = _size(rng, 1, 1 << 20), _size(rng, 16, 1024), _size(rng, 2000, 141000)
            if rows * width <= (1 << 29) // (2 if dtype == "f32" else 1):
                return _embed(None, dtype, way, rows, width, vocab)
    if op == "recur":
        joint, state = rng.random() < 0.5, rng.random() < 0.5
        if rng.random() < 0.25:
            return _recur(None, dtype, "step", _size(rng, 1, 8192), _size(rng, 16, 2048), 1, joint, True)
        while True:
            rows, width = _size(rng, 1, 262144), _size(rng, 16, 2048)
            cost = (2 if dtype == "f32" else 1) * (4 if way == "train" else 1)
            if rows * width * cost <= 262144 * 1000:
                docs = _log_int(rng, 1, max(1, rows // 8))
                return _recur(None, dtype, way, rows, width, docs, joint, state)
    slow = 16 if dtype == "f32" else 1  # matrix products in single precision run at a sixteenth of the rate
    while True:
        rows, width, vocab = _size(rng, 1, 8192), _size(rng, 16, 1024), _size(rng, 2000, 141000)
        if rows * width * vocab * slow <= 8192 * 1024 * 141000:
            return _distill(None, dtype, way, rows, width, vocab, _log_int(rng, 1, 128), rng.random() < 0.5,
                            rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]))


def _zipf(vocab):
    """Cumulative frequencies of words that follow a Zipf law."""
    freq = 1.0 / torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** 1.07
    return torch.cumsum(freq / freq.sum(), 0)


def prepare(case, seed):
    dtype = _DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)

    def normal(*shape, scale=1.0, shift=0.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(to)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float64)

    rows, width = case["rows"], case["width"]
    s = dict(case=case)
    if case["op"] == "embed":
        vocab = case["vocab"]
        # words follow a Zipf law, in no order of frequency; one in fifty places is padding
        name = torch.randperm(vocab, generator=gen, device="cuda")
        word = name[torch.searchsorted(_zipf(vocab), uniform(rows)).clamp_(max=vocab - 1)].to(torch.int32)
        pad = uniform(rows) < 0.02
        pad[0] = False
        s["words"] = torch.where(pad, torch.full_like(word, -1), word)
        s["weight"] = normal(vocab, width, scale=width ** -0.5)
        s["scale"] = width ** 0.5
        s["dy"] = normal(rows, width, scale=0.1)
    elif case["op"] == "recur":
        # some channels forget within a few words, some keep a whole document
        level = 2.0 * torch.randn(width, generator=gen, device="cuda") + 2.0
        both = torch.cat([normal(rows, width), (torch.randn(rows, width, generator=gen, device="cuda") + level).to(dtype)],
                         1)
        s["x"], s["gate"] = both[:, :width], both[:, width:]
        if not case["joint"]:
            s["x"], s["gate"] = s["x"].contiguous(), s["gate"].contiguous()
        if case["way"] == "step":
            s["state"] = normal(rows, width, to=torch.float32)
            return s
        docs = case["docs"]
        # lengths as they fall, empty documents among them; a few rows behind the last one are padding
        end = rows - (rows // 100 if docs > 1 else 0)
        cuts = torch.sort((uniform(docs - 1) * (end + 1)).long().clamp_(max=end)).values
        ends = torch.tensor([0, end], device="cuda")
        s["offsets"] = torch.cat([ends[:1], cuts, ends[1:]])
        s["longest"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
        s["state"] = normal(docs, width, to=torch.float32) if case["state"] else None
        s["dh"] = normal(rows, width)
        s["dlast"] = normal(docs, width, to=torch.float32)
    else:
        vocab, top = case["vocab"], case["top"]
        s["x"] = normal(rows, width)
        s["weight"] = normal(vocab, width, scale=width ** -0.5)
        cdf = _zipf(vocab)
        freq = torch.diff(cdf, prepend=cdf.new_zeros(1))
        s["bias"] = torch.log(freq).to(torch.float32) if case["bias"] else None
        # the teacher's words: one from each of `top` equal shares of the frequencies, each word once, so that a list
        # may be shorter than its row (empty places hold -1)
        place = (torch.arange(top, device="cuda") + uniform(rows, top)) / top
        word = torch.searchsorted(cdf, place).clamp_(max=vocab - 1)
        word[:, 1:][word[:, 1:] == word[:, :-1]] = -1
        # a twentieth of the rows have no teacher
        pad = uniform(rows) < 0.05
        pad[0] = False
        word[pad] = -1
        s["words"] = word.to(torch.int32)
        s["scores"] = normal(rows, top, scale=1.5, shift=-3.0, to=torch.float32)
        s["temperature"] = case["temperature"]
        s["dloss"] = (0.5 + uniform(rows)).float() / rows * (1024.0 if case["dtype"] == "f16" else 1.0)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2007_08725_amd import ops

    case = s["case"]
    train = case["way"] == "train"
    if case["op"] == "embed":
        out = dict(y=ops.embedding(s["words"], s["weight"], s["scale"]))
        if train:
            out["dweight"] = ops.embedding_backward(s["dy"], s["words"], case["vocab"], s["scale"])
        return out
    if case["op"] == "recur":
        if case["way"] == "step":
            h, state = ops.recurrence_step(s["x"], s["gate"], s["state"])
            return dict(h=h, state=state)
        h, last, kept = ops.recurrence(s["x"], s["gate"], s["offsets"], s["state"])
        out = dict(h=h, last=last)
        if train:
            dx, dgate, dstate = ops.recurrence_backward(s["dh"], s["x"], s["gate"], s["offsets"], kept, s["state"],
                                                        s["dlast"])
            out.update(dx=dx, dgate=dgate)
            if dstate is not None:
                out["dstate"] = dstate
        return out
    given = s["x"], s["weight"], s["words"], s["scores"], s["bias"], s["temperature"]
    loss, lse, logits = ops.softmax_distill(*given)
    out = dict(loss=loss, lse=lse, logits=logits)
    if train:
        dx, dweight, dbias = ops.softmax_distill_backward(s["dloss"], lse, logits, *given)
        out.update(dx=dx, dweight=dweight)
        if dbias is not None:
            out["dbias"] = dbias
    return out


def _run_plain(s):
    case = s["case"]
    if case["op"] == "embed":
        return _plain_embed(s, case)
    if case["op"] == "recur":
        return _plain_step(s, case) if case["way"] == "step" else _plain_recur(s, case)
    return _plain_distill(s, case)


def _plain_embed(s, case):
    dtype = _DTYPES[case["dtype"]]
    words, w = s["words"], s["weight"]
    kept = ((words >= 0) & (words < case["vocab"]))[:, None]
    at = words.clamp(0, case["vocab"] - 1).long()
    out = dict(y=torch.where(kept, w[at].float() * s["scale"], torch.zeros((), device=w.device)).to(dtype))
    if case["way"] == "train":
        dy = torch.where(kept, s["dy"].float(), torch.zeros((), device=w.device))
        if dtype == torch.float32:
            # a frequent word's sum may have a hundred thousand terms, which takes more bits than single precision has:
            # sorted by word, running sums in 64 bits, and their differences between a word's first and last place
            names, order = torch.sort(at, stable=True)
            total = torch.cumsum(dy[order].t().contiguous().double(), 1)
            total = torch.cat([torch.zeros_like(total[:, :1]), total], 1)
            places = torch.searchsorted(names, torch.arange(case["vocab"] + 1, device=w.device))
            dw = (total[:, places[1:]] - total[:, places[:-1]]).t()
        else:
            dw = torch.zeros(w.shape, device=w.device).index_add_(0, at, dy)
        out["dweight"] = (dw * s["scale"]).to(dtype)
    return out


def _gates(gate):
    """The sigmoid and one minus it, neither from the other."""
    return 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))


def _plain_step(s, case):
    f, keep = _gates(s["gate"].float())
    state = f * s["state"] + keep * s["x"].float()
    return dict(h=state.to(_DTYPES[case["dtype"]]), state=state)


def _scan(a, b, longest):
    """b_t + a_t b_{t-1} + a_t a_{t-1} b_{t-2} + ..: in steps that double the reach, for chains of at most ``longest``."""
    reach = 1
    while reach < longest:
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _plain_recur(s, case):
    dtype = _DTYPES[case["dtype"]]
    offsets, docs, rows = s["offsets"], case["docs"], case["rows"]
    row = torch.arange(rows, device=offsets.device)
    doc = (torch.searchsorted(offsets, row, right=True) - 1).clamp(max=docs - 1)
    inside = (row < offsets[-1])[:, None]
    first = (row == offsets[doc])[:, None]
    full = torch.nonzero(offsets[1:] > offsets[:-1])[:, 0]  # documents with words
    begin, end = offsets[:-1][full], offsets[1:][full] - 1
    x = s["x"].float()
    f, keep = _gates(s["gate"].float())
    zero = torch.zeros((), device=x.device)
    b = torch.where(inside, keep * x, zero)
    if s["state"] is not None:
        b[begin] += f[begin] * s["state"][full]
    a = torch.where(first | ~inside, zero, f)
    h = _scan(a, b, s["longest"])
    last = s["state"].clone() if s["state"] is not None else torch.zeros(docs, x.shape[1], device=x.device)
    last[full] = h[end]
    out = dict(h=h.to(dtype), last=last)
    if case["way"] == "train":
        g = torch.where(inside, s["dh"].float(), zero)
        g[end] += s["dlast"][full]
        # backwards in time: a row's gradient takes the next row's, times that row's gate
        nxt = torch.cat([a[1:], torch.zeros_like(a[:1])])
        g = _scan(nxt.flip(0), g.flip(0), s["longest"]).flip(0)
        before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
        before = torch.where(first, zero, before)
        if s["state"] is not None:
            before[begin] = s["state"][full]
            dstate = s["dlast"].clone()
            dstate[full] = (f * g)[begin]
            out["dstate"] = dstate
        out["dx"] = (keep * g).to(dtype)
        out["dgate"] = torch.where(inside, g * (before - x) * f * keep, zero).to(dtype)
    return out


def _plain_distill(s, case):
    dtype = _DTYPES[case["dtype"]]
    x, w = s["x"].float(), s["weight"].float()
    words, t = s["words"], s["temperature"]
    there = (words >= 0) & (words < case["vocab"])
    kept = there.any(1)
    at = words.clamp(0, case["vocab"] - 1).long()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"]
    z = z / t
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    zero = torch.zeros((), device=x.device)
    score = torch.where(there, s["scores"] / t, torch.full((), -math.inf, device=x.device))
    high = torch.where(kept, score.max(1).values, zero)[:, None]
    p = torch.exp(score - high)
    mass = torch.where(kept, p.sum(1), zero + 1)[:, None]
    p = p / mass
    logits = torch.where(there, z.gather(1, at), zero)
    apart = (score - high - torch.log(mass)) - (logits - lse[:, None])
    loss = torch.where(there & (p > 0), p * apart, zero).sum(1)
    out = dict(loss=torch.where(kept, loss, zero), lse=lse, logits=logits)
    if case["way"] == "train":
        g = (e / total).scatter_add_(1, at, -p)
        g = g * torch.where(kept, s["dloss"] / t, zero)[:, None]
        out.update(dx=(g @ w).to(dtype), dweight=(g.t() @ x).to(dtype))
        if s["bias"] is not None:
            out["dbias"] = g.sum(0)
    return out


def _distinct(draws, vocab):
    """Expected number of words among ``draws`` of a Zipf law."""
    freq = 1.0 / torch.arange(1, vocab + 1, dtype=torch.float64) ** 1.07
    return int((1 - torch.exp(draws * torch.log1p(-freq / freq.sum()))).sum())


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    train = case["way"] == "train"
    n, d = case["rows"], case["width"]
    if case["op"] == "embed":
        # the words, the rows of the table that they name, y; then dy and the table's gradient
        byte = 4 * n + size * d * (_distinct(n, case["vocab"]) + n)
        if train:
            byte += size * d * (n + case["vocab"])
        return dict(bytes=byte, flops=n * d * (2 if train else 1))
    if case["op"] == "recur":
        if case["way"] == "step":
            return dict(bytes=n * d * (3 * size + 8), flops=10 * n * d)
        # x, gate, h, the documents' last states; then dh, dx, dgate and the states' gradients
        byte = n * d * size * (6 if train else 3) + 8 * (case["docs"] + 1)
        byte += 4 * case["docs"] * d * ((2 if train else 1) * (2 if case["state"] else 1))
        return dict(bytes=byte, flops=n * d * (22 if train else 10))
    v, k = case["vocab"], case["top"]
    # x, the weights, the teacher's words and scores, loss, lse, logits; then dloss and the gradients
    byte = size * (n * d + v * d) * (2 if train else 1) + n * k * 12 + n * (12 if train else 8)
    if case["bias"]:
        byte += 4 * v * (2 if train else 1)
    return dict(bytes=byte, flops=2 * n * d * v * (3 if train else 1))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        return _exact_embed(s, case)
    if case["op"] == "recur":
        if case["way"] == "step":
            gate = s["gate"].double()
            state = torch.lerp(s["x"].double(), s["state"].double(), torch.special.expit(gate))
            return dict(h=state, state=state)
        return _exact_recur(s, case)
    return _exact_distill(s, case)


def _exact_embed(s, case):
    f8 = torch.float64
    vocab = case["vocab"]
    words = s["words"].long()
    table = torch.cat([s["weight"].to(f8) * s["scale"], torch.zeros(1, case["width"], dtype=f8, device=words.device)])
    names = torch.where((words < 0) | (words >= vocab), torch.full_like(words, vocab), words)
    out = dict(y=torch.index_select(table, 0, names))
    if case["way"] == "train":
        dw = torch.zeros(vocab + 1, case["width"], dtype=f8, device=words.device)
        # the words' places in turn, so that few of them wait for one row at a time
        for i in range(16):
            dw.index_add_(0, names[i::16], s["dy"][i::16].to(f8))
        dw = dw[:vocab] * s["scale"]
        out["dweight"] = dw
    return out


def _blockwise(a, b, back=False, block=256):
    """y_t = a_t y_{t-1} + b_t (y_{t+1} with ``back``): row after row inside blocks, all blocks at once, then block
    after block."""
    rows, width = b.shape
    blocks = -(-rows // block)
    a, b = (torch.cat([t, t.new_zeros(blocks * block - rows, width)]).view(blocks, block, width) for t in (a, b))
    y, p = torch.empty_like(b), torch.empty_like(a)
    order = range(block - 1, -1, -1) if back else range(block)
    prev = one = None
    for j in order:
        y[:, j] = b[:, j] if prev is None else a[:, j] * y[:, prev] + b[:, j]
        p[:, j] = a[:, j] if prev is None else a[:, j] * one
        prev, one = j, p[:, j]
    carry = torch.zeros(width, dtype=b.dtype, device=b.device)
    for i in (range(blocks - 1, -1, -1) if back else range(blocks)):
        y[i] += p[i] * carry
        carry = y[i, 0 if back else block - 1].clone()
    return y.view(blocks * block, width)[:rows]


def _exact_recur(s, case):
    f8 = torch.float64
    bounds = s["offsets"].tolist()
    docs, rows, width = case["docs"], case["rows"], case["width"]
    some = [i for i in range(docs) if bounds[i + 1] > bounds[i]]
    index = torch.tensor(some, dtype=torch.long, device=s["x"].device)
    begin = torch.tensor([bounds[i] for i in some], dtype=torch.long, device=s["x"].device)
    end = torch.tensor([bounds[i + 1] - 1 for i in some], dtype=torch.long, device=s["x"].device)
    pad = bounds[-1]
    x = s["x"].to(f8)
    gate = s["gate"].to(f8)
    f, rest = torch.special.expit(gate), torch.special.expit(-gate)
    start = (s["state"] if s["state"] is not None else torch.zeros(docs, width, device=x.device)).to(f8)
    link = f.clone()
    link[begin] = 0
    link[pad:] = 0
    b = rest * x
    b[pad:] = 0
    b[begin] = f[begin] * start[index] + b[begin]
    h = _blockwise(link, b)
    last = start.clone()
    last[index] = h[end]
    out = dict(h=h, last=last)
    if case["way"] == "train":
        g = s["dh"].to(f8)
        g[pad:] = 0
        g[end] += s["dlast"].to(f8)[index]
        g = _blockwise(torch.roll(link, -1, 0), g, back=True)
        before = torch.roll(h, 1, 0)
        before[begin] = start[index]
        out["dx"] = rest * g
        dgate = g * (before - x) * (f * rest)
        dgate[pad:] = 0
        out["dgate"] = dgate
        if s["state"] is not None:
            dstart = s["dlast"].to(f8)
            dstart[index] = g[begin] * f[begin]
            out["dstate"] = dstart
    return out


def _exact_distill(s, case):
    f8 = torch.float64
    n, v, t = case["rows"], case["vocab"], s["temperature"]
    x, w = s["x"].to(f8), s["weight"].to(f8)
    wt = w.T.contiguous()
    words = s["words"].long()
    loss, lse = (torch.zeros(n, dtype=f8, device=x.device) for _ in range(2))
    logits = torch.zeros(words.shape, dtype=f8, device=x.device)
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(v, dtype=f8, device=x.device)
    # a thousand rows at a time: the logits of a whole batch in 64 bits take gigabytes
    for i in range(0, n, 1024):
        part = slice(i, min(n, i + 1024))
        z = torch.mm(x[part], wt)
        if s["bias"] is not None:
            z += s["bias"].to(f8)
        z /= t
        lse[part] = torch.logsumexp(z, 1)
        rows, slots = torch.nonzero((words[part] >= 0) & (words[part] < v), as_tuple=True)
        at = words[part][rows, slots]
        # the teacher's logarithms over its own words
        score = torch.full(words[part].shape, -math.inf, dtype=f8, device=x.device)
        score[rows, slots] = s["scores"][part].to(f8)[rows, slots] / t
        log_p = (score - torch.logsumexp(score, 1, keepdim=True))[rows, slots]
        p = torch.exp(log_p)
        logits[part][rows, slots] = z[rows, at]
        loss[part].index_add_(0, rows, p * (log_p - z[rows, at] + lse[part][rows]))
        if case["way"] == "train":
            g = torch.exp(z - lse[part][:, None])
            g.index_put_((rows, at), -p, accumulate=True)
            has = torch.zeros(g.shape[0], dtype=torch.bool, device=x.device)
            has[rows] = True
            g *= torch.where(has, s["dloss"][part].to(f8) / t, torch.zeros((), dtype=f8, device=x.device))[:, None]
            dx[part] = torch.mm(g, w)
            dw += torch.mm(g.T.contiguous(), x[part])
            db += g.sum(0)
    out = dict(loss=loss, lse=lse, logits=logits)
    if case["way"] == "train":
        out.update(dx=dx, dweight=dw)
        if s["bias"] is not None:
            out["dbias"] = db
    return out
