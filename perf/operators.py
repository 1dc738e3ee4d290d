"""Measured cases of the word-model operators: layer norm, the gated block and
the softmax cross entropy over a vocabulary, forward and with their gradients.

A word model predicts the words of a document from its topic vector: the vector
(one value per topic, or a hidden width) is normalised, goes through a gated
layer, and a softmax over the whole vocabulary scores every token.  A case is
one operator on one shape:

  pass = "forward"  scoring: the operator's outputs alone
  pass = "train"    forward, then the backward pass for a given gradient

Widths are the topic counts that this repository fits (16, 1,000, 32,768),
hidden widths of powers of two and odd sizes between; vocabularies are those of
its corpora (2,000, 102,000, 141,000).  Where ``own`` is false the operators are
computed in their plain form (elementary torch operations in 32 bits), else by
the library's kernels.  ``exact`` gives the definitions in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5


def _norm(name, dtype, way, rows, cols):
    return _named(name, dict(op="norm", dtype=dtype, way=way, rows=rows, cols=cols))


def _gated(name, dtype, way, rows, width, hidden, act="silu"):
    return _named(name, dict(op="gated", dtype=dtype, way=way, rows=rows, width=width, hidden=hidden, act=act))


def _xent(name, dtype, way, rows, width, vocab, bias):
    return _named(name, dict(op="xent", dtype=dtype, way=way, rows=rows, width=width, vocab=vocab, bias=bias))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the topic vector of one document is normalised while it is served: latency alone
        _norm("norm_one_document", "bf16", "forward", 1, 1000),
        # a training batch of hidden states
        _norm("norm_batch", "bf16", "train", 8192, 1024),
        # ragged: a small batch of odd width in single precision
        _norm("norm_odd_f32", "f32", "train", 777, 1013),
        # the widest topic vectors (32,768 topics)
        _norm("norm_wide_f16", "f16", "train", 4096, 32768),
        # one document through the gated layer in serving
        _gated("gated_one_document", "bf16", "forward", 1, 1000, 1024),
        # a training batch
        _gated("gated_batch", "bf16", "train", 8192, 1024, 4096),
        # ragged, in single precision
        _gated("gated_odd_f32", "f32", "train", 517, 1013, 771),
        # scoring a batch of documents by their topics in half precision
        _gated("gated_score_f16", "f16", "forward", 2048, 1000, 2000, "gelu"),
        # one token scored against the largest vocabulary of the benchmarks
        _xent("xent_one_token", "bf16", "forward", 1, 1024, 141000, True),
        # a training batch against the largest vocabulary
        _xent("xent_batch", "bf16", "train", 8192, 1024, 141000, True),
        # a small corpus in single precision, odd width, every size ragged
        _xent("xent_small_f32", "f32", "train", 387, 257, 2000, False),
        # a training batch of a news-sized vocabulary in half precision
        _xent("xent_news_f16", "f16", "train", 4096, 512, 102000, False),
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
    op = rng.choice(["norm", "gated", "gated", "xent", "xent"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    way = rng.choice(["forward", "train", "train"])
    if op == "norm":
        while True:
            rows, cols = _size(rng, 1, 16384), _size(rng, 16, 32768)
            if rows * cols <= 4096 * 32768 // (2 if dtype == "f32" else 1):
                return _norm(None, dtype, way, rows, cols)
    slow = 16 if dtype == "f32" else 1  # matrix products in single precision run at a sixteenth of the rate
    if op == "gated":
        while True:
            rows, width, hidden = _size(rng, 1, 8192), _size(rng, 16, 4096), _size(rng, 16, 4096)
            if rows * width * hidden * slow <= 8192 * 1024 * 4096:
                return _gated(None, dtype, way, rows, width, hidden, rng.choice(["silu", "silu", "gelu", "sigmoid"]))
    while True:
        rows, width, vocab = _size(rng, 1, 8192), _size(rng, 16, 1024), _size(rng, 2000, 141000)
        if rows * width * vocab * slow <= 8192 * 1024 * 141000:
            return _xent(None, dtype, way, rows, width, vocab, rng.random() < 0.5)


def prepare(case, seed):
    dtype = _DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(to)

    rows = case["rows"]
    s = dict(case=case)
    if case["op"] == "norm":
        cols = case["cols"]
        # rows of unlike size and offset, as topic vectors of short and long documents are
        level = torch.randn(rows, 1, generator=gen, device="cuda")
        s["x"] = (torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(0.5 * level) + 0.5 * level).to(dtype)
        s["weight"] = (1 + 0.2 * torch.randn(cols, generator=gen, device="cuda")).to(dtype)
        s["bias"] = normal(cols, scale=0.1)
        s["dy"] = normal(rows, cols)
    elif case["op"] == "gated":
        width, hidden = case["width"], case["hidden"]
        s["x"] = normal(rows, width)
        s["w_gate"] = normal(hidden, width, scale=width ** -0.5)
        s["w_value"] = normal(hidden, width, scale=width ** -0.5)
        s["dh"] = normal(rows, hidden)
    else:
        width, vocab = case["width"], case["vocab"]
        s["x"] = normal(rows, width)
        s["weight"] = normal(vocab, width, scale=width ** -0.5)
        # words follow a Zipf law; the bias is the logarithm of their frequency
        freq = 1.0 / torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** 1.07
        freq = freq / freq.sum()
        s["bias"] = torch.log(freq).to(torch.float32) if case["bias"] else None
        u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)
        label = torch.searchsorted(torch.cumsum(freq, 0), u).clamp_(max=vocab - 1).to(torch.int32)
        # a twentieth of the rows are padding
        pad = torch.rand(rows, generator=gen, device="cuda") < 0.05
        pad[0] = False
        s["labels"] = torch.where(pad, torch.full_like(label, -1), label)
        # a (document, word) pair counts as often as its word occurs there; losses are scaled in half precision
        times = 1 + torch.floor(-torch.log(torch.rand(rows, generator=gen, device="cuda").clamp_(min=1e-6)))
        s["dloss"] = times / rows * (1024.0 if case["dtype"] == "f16" else 1.0)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2007_08725_amd import ops

    case = s["case"]
    train = case["way"] == "train"
    if case["op"] == "norm":
        y, mean, rstd = ops.layer_norm(s["x"], s["weight"], s["bias"], _EPS)
        if not train:
            return dict(y=y)
        dx, dweight, dbias = ops.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd)
        return dict(y=y, dx=dx, dweight=dweight, dbias=dbias)
    if case["op"] == "gated":
        h = ops.gated(s["x"], s["w_gate"], s["w_value"], case["act"])
        if not train:
            return dict(h=h)
        dx, dw_gate, dw_value = ops.gated_backward(s["dh"], s["x"], s["w_gate"], s["w_value"], case["act"])
        return dict(h=h, dx=dx, dw_gate=dw_gate, dw_value=dw_value)
    loss, lse = ops.softmax_xent(s["x"], s["weight"], s["labels"], s["bias"])
    if not train:
        return dict(loss=loss, lse=lse)
    dx, dweight, dbias = ops.softmax_xent_backward(s["dloss"], lse, s["x"], s["weight"], s["labels"], s["bias"])
    out = dict(loss=loss, lse=lse, dx=dx, dweight=dweight)
    if dbias is not None:
        out["dbias"] = dbias
    return out


def _gate(act, a):
    """The gate's activation and its derivative, in the type of a."""
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * phi, phi + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-a))
    if act == "sigmoid":
        return sig, sig * (1 - sig)
    return a * sig, sig * (1 + a * (1 - sig))


def _run_plain(s):
    case = s["case"]
    dtype = _DTYPES[case["dtype"]]
    train = case["way"] == "train"
    x = s["x"].float()
    if case["op"] == "norm":
        w = s["weight"].float()
        c = x - x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + _EPS)
        xh = c * rstd
        out = dict(y=(xh * w + s["bias"].float()).to(dtype))
        if train:
            dy = s["dy"].float()
            g = dy * w
            dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
            out.update(dx=dx.to(dtype), dweight=(dy * xh).sum(0).to(dtype), dbias=dy.sum(0).to(dtype))
        return out
    if case["op"] == "gated":
        wg, wv = s["w_gate"].float(), s["w_value"].float()
        a, b = x @ wg.t(), x @ wv.t()
        p, dp = _gate(case["act"], a)
        out = dict(h=(p * b).to(dtype))
        if train:
            dh = s["dh"].float()
            da, db = dh * b * dp, dh * p
            out.update(dx=(da @ wg + db @ wv).to(dtype), dw_gate=(da.t() @ x).to(dtype),
                       dw_value=(db.t() @ x).to(dtype))
        return out
    w = s["weight"].float()
    rows = torch.arange(x.shape[0], device=x.device)
    kept = s["labels"] >= 0
    label = s["labels"].clamp(min=0).long()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"]
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    out = dict(loss=torch.where(kept, lse - z[rows, label], torch.zeros_like(lse)), lse=lse)
    if train:
        g = e / total
        g[rows, label] -= 1
        g = g * torch.where(kept, s["dloss"], torch.zeros_like(s["dloss"]))[:, None]
        out.update(dx=(g @ w).to(dtype), dweight=(g.t() @ x).to(dtype))
        if s["bias"] is not None:
            out["dbias"] = g.sum(0)
    return out


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    train = case["way"] == "train"
    n = case["rows"]
    if case["op"] == "norm":
        c = case["cols"]
        # x and y; then dy and dx, and the parameters and their gradients
        return dict(bytes=size * (n * c * (4 if train else 2) + c * (4 if train else 2)),
                    flops=n * c * (19 if train else 8))
    if case["op"] == "gated":
        d, f = case["width"], case["hidden"]
        # x, both weights, h; then dh, dx and the weights' gradients
        return dict(bytes=size * (n * d + 2 * f * d + n * f) * (2 if train else 1), flops=4 * n * d * f * (3 if train else 1))
    d, v = case["width"], case["vocab"]
    byte = size * (n * d + v * d) * (2 if train else 1) + n * (4 + 8) + (4 * n if train else 0)
    if case["bias"]:
        byte += 4 * v * (2 if train else 1)
    return dict(bytes=byte, flops=2 * n * d * v * (3 if train else 1))


def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    train = case["way"] == "train"
    x = s["x"].to(f8)
    n = x.shape[0]
    if case["op"] == "norm":
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        sd = torch.sqrt(var + _EPS)
        x = (x - mean) / sd
        out = dict(y=torch.addcmul(s["bias"].to(f8), x, s["weight"].to(f8)))
        if train:
            dy = s["dy"].to(f8)
            out["dweight"], out["dbias"] = (x * dy).sum(0), dy.sum(0)
            g = dy * s["weight"].to(f8)
            # the projections of g on the constant row and on the normalised row go
            g = g - g.mean(1, keepdim=True)
            out["dx"] = (g - x * (g * x).mean(1, keepdim=True)) / sd
        return out
    if case["op"] == "gated":
        wg, wv = s["w_gate"].to(f8), s["w_value"].to(f8)
        a, b = torch.mm(x, wg.T), torch.mm(x, wv.T)
        act = case["act"]
        if act == "gelu":
            half = torch.special.ndtr(a)
            p, dp = a * half, half + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
        else:
            sig = torch.special.expit(a)
            p, dp = (sig, sig * torch.special.expit(-a)) if act == "sigmoid" else (a * sig, sig + a * sig * torch.special.expit(-a))
        out = dict(h=p * b)
        if train:
            dh = s["dh"].to(f8)
            both = torch.cat([dh * b * dp, dh * p], 1)
            dw = torch.mm(both.T.contiguous(), x)
            f = wg.shape[0]
            out.update(dx=torch.mm(both, torch.cat([wg, wv], 0)), dw_gate=dw[:f], dw_value=dw[f:])
        return out
    # a thousand rows at a time: the logits of a whole batch in 64 bits take tens of gigabytes
    w = s["weight"].to(f8)
    wt = w.T.contiguous()
    label = s["labels"].long()
    loss, lse = torch.zeros(n, dtype=f8, device=x.device), torch.empty(n, dtype=f8, device=x.device)
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(w.shape[0], dtype=f8, device=x.device)
    for i in range(0, n, 1024):
        part = slice(i, min(n, i + 1024))
        z = torch.mm(x[part], wt)
        if s["bias"] is not None:
            z += s["bias"].to(f8)
        lse[part] = torch.logsumexp(z, 1)
        kept = torch.nonzero(label[part] >= 0)[:, 0]
        at = label[part][kept]
        loss[i + kept] = lse[part][kept] - z[kept, at]
        if train:
            g = torch.zeros_like(z)
            g[kept] = torch.exp(z[kept] - lse[part][kept, None])
            g[kept, at] -= 1
            g *= s["dloss"][part].to(f8)[:, None]
            dx[part] = torch.mm(g, w)
            dw += torch.mm(g.T.contiguous(), x[part])
            db += g.sum(0)
    out = dict(loss=loss, lse=lse)
    if train:
        out.update(dx=dx, dweight=dw)
        if s["bias"] is not None:
            out["dbias"] = db
    return out
