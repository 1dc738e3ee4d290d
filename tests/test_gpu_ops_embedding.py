"""Word embedding (include/lda_ops.h) against its formulas in 64 bits; bounds as in test_gpu_ops.py: a product is off by
E of itself, a sum of n terms by g(n) of their magnitudes, and an output by half a step of its type."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, TYPES, check, directional, g, ops, rand, strided, STEP, ROOM  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def words_of(seed, rows, vocab, low=0, high=None):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(low, vocab if high is None else high, (rows,), generator=gen, dtype=torch.int32).cuda()


def skewed(seed, rows, vocab):
    """A third of the rows one word, the others spread."""
    w = words_of(seed, rows, vocab)
    w[torch.arange(rows, device="cuda") % 3 == 1] = vocab // 2
    return w


def case(ops, dtype, words, vocab, width, scale, pad=0, offset=0):  # noqa: F811
    rows = words.shape[0]
    weight = strided(rand(1, vocab, width, dtype=dtype), pad, offset)
    dy = strided(rand(2, rows, width, dtype=dtype), pad, offset)
    kept = ((words >= 0) & (words < vocab))[:, None]
    at = words.long().clamp(0, vocab - 1)
    want = torch.where(kept, weight.to(F8)[at] * scale, torch.zeros((), dtype=F8, device="cuda"))
    # the scale is rounded to 32 bits, and so is the product
    check("y", ops.embedding(words, weight, scale), want, 2 * E * want.abs())
    dw = ops.embedding_backward(dy, words, vocab, scale)
    d8 = torch.where(kept, dy.to(F8), torch.zeros((), dtype=F8, device="cuda"))
    total, size = (torch.zeros(vocab, width, dtype=F8, device="cuda").index_add_(0, at, t) for t in (d8, d8.abs()))
    most = int(torch.bincount(at).max()) if rows else 0
    check("dweight", dw, total * scale, (g(most) + 2 * E) * size * abs(scale))
    absent = torch.ones(vocab, dtype=torch.bool, device="cuda")
    absent[at[kept[:, 0]]] = False
    assert not bool(dw[absent].any())


# one piece, several, words over the ends of pieces; the sort in one workgroup (to 8,192 rows) and by digits
SHAPES = [(1, 1, 1), (1, 5, 3), (2, 1000, 7), (63, 16, 40), (64, 17, 9), (65, 64, 64), (128, 8, 1), (129, 300, 33),
          (1000, 257, 50), (1025, 40, 3), (4097, 24, 2000), (8192, 16, 999), (8193, 16, 511), (8193, 33, 512),
          (20001, 72, 141000), (30000, 5, 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,vocab", SHAPES)
def test_embedding(ops, dtype, rows, width, vocab):  # noqa: F811
    case(ops, dtype, skewed(rows, rows, vocab), vocab, width, 1.0 if rows % 2 else 16.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 2, 6, 30, 64, 514, 1024, 1500])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1), (8, 8), (2, 2)])
def test_embedding_widths_and_strides(ops, dtype, width, pad, offset):  # noqa: F811
    case(ops, dtype, words_of(7, 700, 90), 90, width, -0.37, pad, offset)


@pytest.mark.parametrize("rows", [50, 9000, 40000])
def test_embedding_words_outside_the_vocabulary(ops, rows):  # noqa: F811
    """Padding at any place, the types' extremes among it; what those rows of dy hold has no part."""
    vocab, width = 70, 24
    words = words_of(3, rows, vocab, -60, vocab + 60)
    words[5], words[6], words[7] = 2 ** 31 - 1, -2 ** 31, vocab
    case(ops, torch.float32, words, vocab, width, 2.0)
    out = (words < 0) | (words >= vocab)
    dy = rand(4, rows, width)
    want = ops.embedding_backward(dy, words, vocab, 2.0)
    dy[out] = float("nan")
    assert torch.equal(want, ops.embedding_backward(dy, words, vocab, 2.0))
    none = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    assert not bool(ops.embedding(none, rand(1, vocab, width)).any())
    assert not bool(ops.embedding_backward(dy, none, vocab).any())


@pytest.mark.parametrize("rows", [64, 65, 1088, 1089, 8192, 70000, 200001])
def test_embedding_one_word_many_times(ops, rows):  # noqa: F811
    """A word whose sum goes through many pieces, alone and after others."""
    for first in (0, 1, 63, 64):
        words = torch.full((rows,), 2, dtype=torch.int32, device="cuda")
        words[:first] = 1
        case(ops, torch.float32, words[torch.randperm(rows, generator=torch.Generator().manual_seed(1)).cuda()], 4, 8,
             1.0)


def test_embedding_words_of_every_count(ops):  # noqa: F811
    """Words of 0, 1, 2, .. 300 rows, so that every length meets every place of a piece's end."""
    count = torch.arange(301)
    words = torch.repeat_interleave(count, count).to(torch.int32)
    words = words[torch.randperm(words.shape[0], generator=torch.Generator().manual_seed(2))].cuda()
    case(ops, torch.float32, words, 301, 20, 1.0)
    case(ops, torch.bfloat16, words, 301, 72, 1.0)


def test_embedding_large_vocabulary(ops):  # noqa: F811
    """The largest word ids: 25 bits of keys, three digits."""
    vocab = ops.MAX_VOCAB
    words = words_of(1, 9001, vocab)
    words[3], words[4] = vocab - 1, vocab
    weight = torch.zeros(vocab, 1, device="cuda")
    weight[:, 0] = torch.arange(vocab, device="cuda")
    kept = words < vocab
    assert torch.equal(ops.embedding(words, weight, 1.0)[:, 0], torch.where(kept, words.float(), torch.zeros(())))
    dw = ops.embedding_backward(torch.ones(9001, 1, device="cuda"), words, vocab)
    assert torch.equal(dw[:, 0], torch.bincount(words[kept].long(), minlength=vocab).float())


def test_embedding_far_offsets(ops):  # noqa: F811
    """Elements beyond 2^32 of y, of dy and of the gradient."""
    rows, width, vocab = 4300000, 1024, 4300000
    words = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0)
    words[5] = vocab - 7  # twice, the word 4299994 not at all
    weight = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    weight[:] = torch.arange(vocab, device="cuda")[:, None] % 251
    y = ops.embedding(words, weight, 2.0)
    want = (words.long() % 251 * 2).to(torch.bfloat16)
    assert bool((y == want[:, None]).all())
    del weight
    dw = ops.embedding_backward(y, words, vocab, 0.5)
    del y
    sums = torch.zeros(vocab, device="cuda").index_add_(0, words.long(), want.float()) * 0.5
    assert bool((dw == sums.to(torch.bfloat16)[:, None]).all())


def test_embedding_empty(ops):  # noqa: F811
    words = torch.empty(0, dtype=torch.int32, device="cuda")
    weight = rand(1, 70, 24, dtype=torch.bfloat16)
    y = ops.embedding(words, weight)
    assert y.shape == (0, 24) and y.dtype == torch.bfloat16
    assert not bool(ops.embedding_backward(y, words, 70).any())


def test_embedding_gradient_against_differences(ops):  # noqa: F811
    weight, c, words = rand(1, 30, 20), rand(2, 100, 20), words_of(3, 100, 33)
    grad = ops.embedding_backward(c, words, 30, 1.5)
    got, want = directional(lambda t: float((ops.embedding(words, t[0], 1.5).to(F8) * c.to(F8)).sum()), [grad],
                            [weight], 10, STEP)
    assert abs(got - want) <= ROOM * max(1.0, abs(want))


def test_embedding_broadcast_and_rows_beside(ops):  # noqa: F811
    """Gradients that are one row in memory; rows beside a strided gradient's columns are not read into it."""
    one = rand(1, 1, 64, dtype=torch.float16)
    words = words_of(2, 3000, 50)
    assert torch.equal(ops.embedding_backward(one.expand(3000, 64), words, 50),
                       ops.embedding_backward(one.expand(3000, 64).contiguous(), words, 50))


def test_embedding_same_bits_and_streams(ops):  # noqa: F811
    words, dy = skewed(1, 60000, 5000), rand(2, 60000, 136, dtype=torch.bfloat16)
    first = ops.embedding_backward(dy, words, 5000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = ops.embedding_backward(dy, words, 5000)
    side.synchronize()
    assert torch.equal(first, second) and torch.equal(first, ops.embedding_backward(dy, words, 5000))


@pytest.mark.parametrize("rows", [300, 30000])
def test_embedding_in_a_graph(ops, rows):  # noqa: F811
    """Captured once, replayed on new words, with the program's own work between."""
    words, dy, weight = words_of(1, rows, 900), rand(2, rows, 40), rand(3, 900, 40)

    def everything():
        return ops.embedding(words, weight, 3.0), ops.embedding_backward(dy, words, 900, 3.0)

    everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for i in range(4):
        words.copy_(words_of(10 + i, rows, 900, -50, 450 + 100 * i))
        dy.copy_(rand(20 + i, rows, 40))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, everything()):
            assert torch.equal(a, b), i


def test_embedding_refusals(ops):  # noqa: F811
    weight, words, dy = rand(1, 8, 16), words_of(2, 4, 8), rand(3, 4, 16)
    bad = [lambda: ops.embedding(words.long(), weight), lambda: ops.embedding(words, weight.double()),
           lambda: ops.embedding(words, weight.t()), lambda: ops.embedding(words[::2], weight),
           lambda: ops.embedding(words, weight[:0]), lambda: ops.embedding(words.cpu(), weight),
           lambda: ops.embedding(words.view(2, 2), weight), lambda: ops.embedding(None, weight),
           lambda: ops.embedding_backward(dy, words[:3], 8), lambda: ops.embedding_backward(dy, words, 0),
           lambda: ops.embedding_backward(dy, words, ops.MAX_VOCAB + 1), lambda: ops.embedding_backward(dy[0], words, 8),
           lambda: ops.embedding(words, weight.clone().requires_grad_())]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d did not come" % i)
    from paper_2007_08725_amd import LDAError
    for scale in (float("nan"), float("inf")):
        with pytest.raises(LDAError):
            ops.embedding(words, weight, scale)
        with pytest.raises(LDAError):
            ops.embedding_backward(dy, words, 8, scale)
