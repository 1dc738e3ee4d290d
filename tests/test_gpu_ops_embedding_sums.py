"""The embedding's gradient in single precision (include/lda_ops.h): a word's sum is off by its own rounding alone,
however many rows the word has and wherever its pieces end.

Sums of n terms in 64 bits are within (n + 8) 2^-53 of their magnitudes' sum, the scale's product within 2^-53 of
itself, and the result is rounded once, by half a step of single precision at most.
"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, TINY, check, ops, rand, strided  # noqa: E402,F401
from test_gpu_ops_embedding import words_of  # noqa: E402

pytestmark = pytest.mark.gpu


def case(ops, words, vocab, dy, scale):  # noqa: F811
    kept = (words >= 0) & (words < vocab)
    at, d8 = words.long()[kept], dy.to(F8)[kept]
    total, size = (torch.zeros(vocab, dy.shape[1], dtype=F8, device="cuda").index_add_(0, at, t)
                   for t in (d8, d8.abs()))
    most = int(torch.bincount(at).max())
    check("dweight", ops.embedding_backward(dy, words, vocab, scale), total * scale,
          (2 * most + 16) * 2.0 ** -53 * size * abs(scale))


# words of hundreds, thousands and a hundred thousand rows; the pieces' lengths go from 16 to 512
@pytest.mark.parametrize("rows,width,vocab", [(700, 5, 2), (5000, 3, 1), (5000, 257, 3), (50000, 40, 7),
                                              (105000, 24, 1), (210000, 1, 2), (1 << 20, 72, 9)])
@pytest.mark.parametrize("scale", [1.0, -0.75])
def test_frequent_words_in_single_precision(ops, rows, width, vocab, scale):  # noqa: F811
    words = words_of(rows, rows, vocab, -1)
    case(ops, words, vocab, strided(rand(2, rows, width), 3, 1), scale)


def test_sums_that_cancel(ops):  # noqa: F811
    """Large values that take each other away leave the small ones between them whole."""
    rows, width = 60000, 16
    dy = rand(1, rows, width)
    big = torch.arange(rows, device="cuda")[:, None] % 3
    dy = torch.where(big == 0, torch.full_like(dy, 2.0 ** 20), torch.where(big == 1, torch.full_like(dy, -2.0 ** 20), dy))
    case(ops, torch.zeros(rows, dtype=torch.int32, device="cuda"), 1, dy, 1.0)
    case(ops, words_of(3, rows, 4), 4, dy, 1.0)


def test_infinities_and_nan_reach_their_word_alone(ops):  # noqa: F811
    rows, width, vocab = 9000, 20, 5
    words, dy = words_of(1, rows, vocab), rand(2, rows, width)
    want = ops.embedding_backward(dy, words, vocab)
    dy[words == 3] = float("inf")
    dy[torch.nonzero(words == 1)[0, 0], 4] = float("nan")
    got = ops.embedding_backward(dy, words, vocab)
    sound = torch.tensor([0, 2, 4], device="cuda")
    assert torch.equal(got[sound], want[sound]) and bool((got[3] == float("inf")).all())
    assert bool(got[1, 4].isnan()) and torch.equal(got[1, 5:], want[1, 5:])


def test_largest_values_do_not_overflow_on_the_way(ops):  # noqa: F811
    """Sums past the type's range that come back into it."""
    dy = torch.tensor([[3e38], [3e38], [-3e38], [-2e38]], device="cuda")
    got = ops.embedding_backward(dy, torch.zeros(4, dtype=torch.int32, device="cuda"), 1)
    assert abs(float(got[0, 0]) / float(dy.to(F8).sum()) - 1) <= E
    many = torch.cat([torch.full((4000, 3), 3e38), torch.full((4000, 3), -3e38), torch.ones(1, 3)]).cuda()
    got = ops.embedding_backward(many, torch.zeros(8001, dtype=torch.int32, device="cuda"), 1)
    assert float((got.to(F8) - many.to(F8).sum(0)).abs().max()) <= 8010 * 2.0 ** -53 * 4000 * 3e38 * 2
