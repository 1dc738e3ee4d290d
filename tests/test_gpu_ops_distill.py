"""Distillation from a teacher's listed words (include/lda_ops.h) against its formulas in 64 bits.

Bounds as in test_gpu_ops.py for the student's softmax (the logits and their
logarithm divided by the temperature).  The teacher's p and its logarithm carry
the scores' rounding, a few E of the largest, and g(top) of the sum.  G of the
16-bit types is rounded once (up to 128 rows what that leaves is kept too, rounded
to the same type: off by U of U); dbias takes the students' and the teachers' parts
in two sums.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, TYPES, U, check, directional, g, ops, rand, strided, STEP, ROOM  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def teacher(seed, rows, vocab, top):
    """Listed words, some places empty (NaN or, in row 0, perhaps listed after all), a row without any, words twice."""
    gen = torch.Generator().manual_seed(seed)
    words = torch.randint(0, vocab, (rows, top), generator=gen, dtype=torch.int32)
    empty = torch.rand(rows, top, generator=gen) < 0.2
    words[empty] = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[
        torch.randint(0, 4, (int(empty.sum()),), generator=gen)]
    words[0, 0] = 0
    if rows > 2:
        words[1] = -1
    if top > 3:
        words[0, 1] = words[0, 3] = 0
    scores = torch.randn(rows, top, generator=gen) * 2 - 3
    scores[empty] = float("nan")
    return words.cuda(), scores.cuda()


def case(ops, dtype, rows, width, vocab, top, with_bias, temperature, pad=0, offset=0, dloss_scale=1.0):  # noqa: F811
    x = strided(rand(1, rows, width, dtype=dtype), pad, offset)
    w = strided(rand(2, vocab, width, scale=2 * width ** -0.5, dtype=dtype), pad, offset)
    bias = rand(3, vocab) if with_bias else None
    words, scores = teacher(4, rows, vocab, top)
    if pad:
        words = torch.cat([words, words], 1)[:, :top]
        scores = strided(scores, pad, offset)
    dloss = rand(5, rows, scale=dloss_scale)
    loss, lse, logits = ops.softmax_distill(x, w, words, scores, bias, temperature)
    x8, w8 = x.to(F8), w.to(F8)
    z = x8 @ w8.t()
    mag = x8.abs() @ w8.abs().t()
    if with_bias:
        z = z + bias.to(F8)
        mag = mag + bias.to(F8).abs()
    z, ez = z / temperature, g(width + 4) * mag / temperature
    there = (words >= 0) & (words < vocab)
    kept = there.any(1)
    at = words.long().clamp(0, vocab - 1)
    rlse = torch.logsumexp(z, 1)
    spread = (z.amax(1) - z.amin(1)).clamp(max=40.0)
    elogit = ez.amax(1)
    elsum = 2 * elogit + 4 * E * spread + 4 * E + g(vocab) + 2 * E * (rlse.abs() + z.abs().amax(1) + math.log(vocab))
    check("lse", lse, rlse, elsum)
    zero = torch.zeros((), dtype=F8, device="cuda")
    listed = torch.where(there, z.gather(1, at), zero)
    check("logits", logits, listed, torch.where(there, ez.gather(1, at), zero))
    s8 = torch.where(there, scores.to(F8) / temperature, zero - math.inf)
    log_p = torch.where(kept[:, None], s8 - torch.logsumexp(s8, 1, keepdim=True), zero - math.inf)
    # a listed NaN is one of its row's listed words, not of its empty places
    p = torch.where(there, torch.exp(log_p), zero)
    most = torch.where(there, s8.abs(), zero).amax(1)
    ep = (E * (12 * most + 40) + g(top))[:, None]  # of p, and of its logarithm
    term = torch.where(there, log_p - (listed - rlse[:, None]), zero)
    eterm = ep + (elogit + elsum)[:, None] + 4 * E * (log_p.clamp(min=-1e3).abs() + listed.abs() + rlse.abs()[:, None])
    check("loss", loss, (p * term).sum(1), (p * (eterm + (ep + g(top)) * term.abs())).sum(1))
    assert not bool(loss[~kept].any())
    dx, dw, db = ops.softmax_distill_backward(dloss, lse, logits, x, w, words, scores, bias, temperature)
    d8 = torch.where(kept, dloss.to(F8), zero)[:, None] / temperature
    q = torch.exp(z - rlse[:, None])
    given = torch.zeros_like(q).scatter_add_(1, at, p)
    egiven = torch.zeros_like(q).scatter_add_(1, at, torch.where(there, p * (ep + top * E), zero))
    grad = d8 * (q - given)
    top_d = float(d8.abs().max())
    u = (0.0 if dtype == torch.float32 else U[dtype] ** 2 if rows <= 128 else U[dtype]) + 6 * E
    eq = q * (2 * elsum + 6 * E * 40 + 2 * elogit)[:, None]
    eg = d8.abs() * (eq + egiven + 2 * E * (q + given)) + u * grad.abs()
    if dtype == torch.float16:
        eg = eg + top_d * 2.0 ** -25 / 2.0 ** 14
    check("dx", dx, grad @ w8, (eg + g(vocab) * grad.abs()) @ w8.abs())
    check("dweight", dw, grad.t() @ x8, (eg + g(rows) * grad.abs()).t() @ x8.abs())
    assert (db is None) == (bias is None)
    if with_bias:
        eb = d8.abs() * (eq + egiven + (6 * E + g(rows) + g(rows * top)) * (q + given))
        check("dbias", db, grad.sum(0), eb.sum(0))


# up to 16 rows and more, one tile and several, one word and the most, vocabularies that end inside a tile
SHAPES = [(1, 1, 1, 1), (1, 16, 2, 2), (1, 1024, 2000, 32), (2, 40, 333, 5), (5, 8, 129, 64), (16, 64, 257, 65),
          (17, 24, 1000, 1), (33, 129, 128, 100), (64, 1013, 300, 20), (100, 257, 2000, 256), (129, 72, 4099, 33),
          (260, 32, 515, 200), (1100, 40, 70, 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab,top", SHAPES)
def test_softmax_distill(ops, dtype, rows, width, vocab, top):  # noqa: F811
    case(ops, dtype, rows, width, vocab, top, (rows + vocab) % 2 == 0, [1.0, 2.0, 0.7][rows % 3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 40])
def test_softmax_distill_words_listed_twice(ops, dtype, rows):  # noqa: F811
    """Places of one word count together: as one place whose p is their sum."""
    vocab = 200
    x, w = rand(1, rows, 32, dtype=dtype), rand(2, vocab, 32, scale=0.2, dtype=dtype)
    bias, dloss = rand(3, vocab), rand(4, rows)
    once = (torch.arange(rows * 3, device="cuda").view(rows, 3) * 11 % vocab).to(torch.int32)
    scores = rand(5, rows, 3)
    twice = torch.cat([once, once, once[:, :1]], 1)
    # a word's places share its probability: log(1/2) each, the first word's three log(1/4), log(1/2), log(1/4)
    share = torch.tensor([[0.25, 0.5, 0.5, 0.5, 0.5, 0.5, 0.25]], device="cuda")
    more = torch.cat([scores, scores, scores[:, :1]], 1) + torch.log(share)
    a = everything(ops, x, w, once, scores, bias, dloss)
    b = everything(ops, x, w, twice, more, bias, dloss)
    assert torch.equal(a[1], b[1])
    # either is a sum of 33 terms in an order of its own: within g(33) of their magnitudes
    size = (x.double().abs() @ w.double().abs().t() + bias.double().abs()).gather(1, once.long())
    for logits in (b[2][:, :3], b[2][:, 3:6]):
        assert bool(((logits - a[2]).double().abs() <= 2 * g(33) * size).all())
    # p is off by some 40 E; so is G, before it is rounded to the type
    room = (80 * E + (U[dtype] if dtype != torch.float32 else 0)) * 2
    for i, many in ((3, vocab), (4, rows), (5, rows)):
        size = float(a[i].abs().max())
        assert float((a[i].double() - b[i].double()).abs().max()) <= room * max(size, 1.0) * 4, i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab,top", [(700, 72, 5003, 16), (2049, 40, 20011, 30), (1030, 257, 9001, 8)])
def test_softmax_distill_larger_tiles(ops, dtype, rows, width, vocab, top):  # noqa: F811
    case(ops, dtype, rows, width, vocab, top, vocab > 9000, 1.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,pad,offset", [(1, 8, 8), (3, 1, 1), (50, 8, 16), (150, 5, 3)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_softmax_distill_strides(ops, dtype, rows, pad, offset, with_bias):  # noqa: F811
    case(ops, dtype, rows, 96, 700, 12, with_bias, 1.0, pad, offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-12, 1e-4, 1e3])
def test_softmax_distill_gradient_scales(ops, dtype, scale):  # noqa: F811
    case(ops, dtype, 60, 64, 900, 9, True, 3.0, dloss_scale=scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_softmax_distill_many_pieces(ops, dtype):  # noqa: F811
    """A vocabulary of several pieces of G, with listed words in each."""
    rows, width, vocab = 3000 if dtype == torch.float32 else 6000, 16, 30011
    case(ops, dtype, rows, width, vocab, 10, True, 1.0)


def everything(ops, x, w, words, scores, bias, dloss, temperature=1.0):  # noqa: F811
    loss, lse, logits = ops.softmax_distill(x, w, words, scores, bias, temperature)
    return [loss, lse, logits, *ops.softmax_distill_backward(dloss, lse, logits, x, w, words, scores, bias, temperature)]


@pytest.mark.parametrize("rows", [12, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_softmax_distill_rows_left_out_may_hold_anything(ops, dtype, rows):  # noqa: F811
    """Rows without listed words, or whose scores are all -inf: no loss, no gradient, whatever x and dloss hold."""
    width, vocab, top = 64, 400, 7
    x, w, bias = rand(1, rows, width, dtype=dtype), rand(2, vocab, width, scale=0.1, dtype=dtype), rand(3, vocab)
    words = (torch.arange(rows * top, device="cuda").view(rows, top) * 13 % vocab).to(torch.int32)
    scores, dloss = rand(4, rows, top), rand(5, rows)
    words[3], scores[5] = -1, -math.inf
    out = torch.zeros(rows, dtype=torch.bool, device="cuda")
    out[3], out[5] = True, True
    want = [t.clone() for t in everything(ops, x, w, words, scores, bias, dloss)]
    x[out], dloss[out], scores[3] = float("nan"), float("inf"), float("nan")
    got = everything(ops, x, w, words, scores, bias, dloss)
    for i, name in ((0, "loss"), (3, "dx"), (4, "dweight"), (5, "dbias")):
        assert torch.equal(got[i], want[i]), name
    assert not bool(got[0][out].any()) and not bool(got[3][out].any())


@pytest.mark.parametrize("rows", [4, 40])
def test_softmax_distill_no_row_kept(ops, rows):  # noqa: F811
    x, w, bias = rand(1, rows, 40), rand(2, 90, 40), rand(3, 90)
    words = torch.full((rows, 5), -1, dtype=torch.int32, device="cuda")
    loss, _, logits, dx, dw, db = everything(ops, x, w, words, rand(4, rows, 5), bias, rand(5, rows))
    for t in (loss, logits, dx, dw, db):
        assert not bool(t.any())


@pytest.mark.parametrize("rows", [4, 40])
def test_softmax_distill_certain_teacher_is_the_cross_entropy(ops, rows):  # noqa: F811
    """One listed word: its loss and its gradients are those of the label, to the roundings of both."""
    x, w, bias = rand(1, rows, 40), rand(2, 300, 40, scale=0.2), rand(3, 300)
    labels = (torch.arange(rows, device="cuda") * 7 % 300).to(torch.int32)
    dloss = rand(4, rows)
    words = torch.full((rows, 3), -1, dtype=torch.int32, device="cuda")
    scores = torch.zeros(rows, 3, device="cuda")
    words[:, 1], words[:, 2], scores[:, 2] = labels, (labels + 1) % 300, -math.inf  # a score of -inf: p = 0
    loss, lse, _, dx, dw, db = everything(ops, x, w, words, scores, bias, dloss)
    loss2, lse2 = ops.softmax_xent(x, w, labels, bias)
    assert torch.equal(lse, lse2)
    want = ops.softmax_xent_backward(dloss, lse2, x, w, labels, bias)
    # the label's logit from another order of 40 terms
    room = 4 * g(40) * float((x.abs() @ w.abs().t()).max() + bias.abs().max())
    assert torch.allclose(loss, loss2, rtol=4 * E, atol=room)
    for a, b in zip((dx, dw, db), want):
        assert torch.allclose(a, b, rtol=0, atol=(room + g(rows + 300)) * 40)


@pytest.mark.parametrize("rows", [4, 40])
def test_softmax_distill_masked_words(ops, rows):  # noqa: F811
    """Words masked by the bias: an unlisted one has no part, a listed one with p > 0 an infinite loss, one with p = 0
    none; the gradients stay finite."""
    x, w, bias = rand(1, rows, 40, scale=0.1), rand(2, 300, 40), rand(3, 300)
    bias[128:256] = -math.inf
    words = torch.tensor([[3, 5, 270]] * rows, dtype=torch.int32, device="cuda")
    scores = rand(4, rows, 3)
    words[1, 1] = 130
    words[2, 1], scores[2, 1] = 131, -math.inf
    loss, lse, logits, dx, dw, db = everything(ops, x, w, words, scores, bias, torch.ones(rows, device="cuda"))
    assert float(loss[1]) == math.inf and float(logits[1, 1]) == -math.inf
    sound = torch.arange(rows, device="cuda") != 1
    assert bool(loss[sound].isfinite().all())
    z = (x.to(F8) @ w.to(F8).t() + bias.to(F8))
    q = torch.softmax(z, 1)
    p = torch.softmax(scores.to(F8), 1)
    grad = q.scatter_add(1, words.long(), -p)
    check("dbias", db, grad.sum(0), g(300) * 8 * torch.ones(300, dtype=F8, device="cuda") * rows)
    check("dx", dx, grad @ w.to(F8), g(300) * 16 * (q + 1) @ w.to(F8).abs())
    only = torch.arange(132, 256, device="cuda")
    assert not bool(dw[only].any()) and not bool(db[only].any())
    bias[:] = -math.inf  # no word left: loss +inf, no gradient
    out = everything(ops, x, w, words, scores, bias, torch.ones(rows, device="cuda"))
    assert bool((out[0] == math.inf).all()) and bool((out[1] == -math.inf).all())
    assert not any(bool(t.any()) for t in out[3:])


def test_softmax_distill_perfect_student_has_no_gradient(ops):  # noqa: F811
    """A teacher that lists every word with the student's own logits: loss and gradients of 0, to the roundings."""
    x, w, bias = rand(1, 30, 24), rand(2, 200, 24, scale=0.2), rand(3, 200)
    words = torch.arange(200, dtype=torch.int32, device="cuda").expand(30, 200).contiguous()
    scores = x @ w.t() + bias
    room = 8 * g(24) * float((x.abs() @ w.abs().t()).max() + bias.abs().max()) + 2 * g(200)
    loss, _, _, dx, dw, db = everything(ops, x, w, words, scores, bias, torch.ones(30, device="cuda"), 1.7)
    assert float(loss.abs().max()) <= room
    for t, many in ((dx, 200), (dw, 30), (db, 30)):
        assert float(t.abs().max()) <= room * many


def test_softmax_distill_empty(ops):  # noqa: F811
    x, w = torch.empty(0, 24, device="cuda"), rand(1, 70, 24)
    words, scores = torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda")
    loss, lse, logits, dx, dw, db = everything(ops, x, w, words, scores, rand(2, 70), torch.empty(0, device="cuda"))
    assert loss.shape == lse.shape == (0,) and logits.shape == (0, 4) and dx.shape == (0, 24)
    assert not bool(dw.any()) and not bool(db.any())


def test_softmax_distill_gradients_against_differences(ops):  # noqa: F811
    x, w, b, c = rand(1, 20, 30), rand(2, 150, 30, scale=0.3), rand(3, 150), rand(4, 20)
    words, scores = teacher(5, 20, 150, 9)
    # row 0 lists a word whose score is NaN: its loss is NaN, and so would be both slopes
    assert bool(scores[0, :4].isnan().any())
    scores = scores.nan_to_num(nan=-1.0)
    grads = everything(ops, x, w, words, scores, b, c, 1.5)[3:]
    got, want = directional(lambda t: float((ops.softmax_distill(t[0], t[1], words, scores, t[2], 1.5)[0].to(F8)
                                             * c.to(F8)).sum()), grads, [x, w, b], 30, STEP)
    assert abs(got - want) <= ROOM * max(1.0, abs(want))


def test_softmax_distill_same_bits_streams_and_graph(ops):  # noqa: F811
    rows, vocab = 500, 3001
    x, w = rand(1, rows, 136, dtype=torch.bfloat16), rand(2, vocab, 136, scale=0.1, dtype=torch.bfloat16)
    bias, dloss = rand(3, vocab), rand(4, rows)
    words, scores = teacher(5, rows, vocab, 40)
    want = everything(ops, x, w, words, scores, bias, dloss, 2.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = everything(ops, x, w, words, scores, bias, dloss, 2.0)
    side.synchronize()
    again = everything(ops, x, w, words, scores, bias, dloss, 2.0)
    for a, b, c in zip(want, other, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything(ops, x, w, words, scores, bias, dloss, 2.0)
    for i in range(4):
        x.copy_(rand(20 + i, rows, 136))
        words.copy_(teacher(30 + i, rows, vocab, 40)[0])
        scores.copy_(rand(40 + i, rows, 40))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, everything(ops, x, w, words, scores, bias, dloss, 2.0)):
            assert torch.equal(a, b), i


def test_softmax_distill_refusals(ops):  # noqa: F811
    x, w, bias, dloss = rand(1, 4, 16), rand(2, 8, 16), rand(3, 8), rand(4, 4)
    words, scores = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), rand(5, 4, 3)
    loss, lse, logits = ops.softmax_distill(x, w, words, scores, bias)
    wide = torch.zeros(4, ops.MAX_TOP + 1, dtype=torch.int32, device="cuda")
    bad = [lambda: ops.softmax_distill(x, w, words.long(), scores), lambda: ops.softmax_distill(x, w, words, scores.half()),
           lambda: ops.softmax_distill(x, w, words[:2], scores[:2]), lambda: ops.softmax_distill(x, w, words, scores[:, :2]),
           lambda: ops.softmax_distill(x, w, words[:, :0], scores[:, :0]),
           lambda: ops.softmax_distill(x, w, wide, wide.float()), lambda: ops.softmax_distill(x, w[:, :8], words, scores),
           lambda: ops.softmax_distill(x, w.half(), words, scores), lambda: ops.softmax_distill(x, w[:0], words, scores),
           lambda: ops.softmax_distill(x, w, words, scores, bias[:4]), lambda: ops.softmax_distill(x, w, None, scores),
           lambda: ops.softmax_distill(x, w, words.cpu(), scores), lambda: ops.softmax_distill(x, w, words, None),
           lambda: ops.softmax_distill(x, w, words, scores.clone().requires_grad_()),
           lambda: ops.softmax_distill_backward(dloss, lse, logits[:, :2], x, w, words, scores, bias),
           lambda: ops.softmax_distill_backward(dloss[:2], lse, logits, x, w, words, scores, bias),
           lambda: ops.softmax_distill_backward(dloss, lse.half(), logits, x, w, words, scores, bias)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d did not come" % i)
    from paper_2007_08725_amd import LDAError
    for temperature in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        with pytest.raises(LDAError):
            ops.softmax_distill(x, w, words, scores, bias, temperature)
        with pytest.raises(LDAError):
            ops.softmax_distill_backward(dloss, lse, logits, x, w, words, scores, bias, temperature)
