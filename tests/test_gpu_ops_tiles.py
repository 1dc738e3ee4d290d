"""The products of the word-model operators at every size of their tiles, against the formulas in 64 bits.

Shapes are such that the choice of tiles (128 x 128 or 64 x 64, 256 x 256 in
16-bit types) and of the parts of a sum takes each form of each product; the
bounds are those of test_gpu_ops.py.
"""
import pytest

from test_gpu_ops import gated_case, ops, rand, xent_case  # noqa: F401 (ops is a fixture)

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

SHORT = [torch.bfloat16, torch.float16]
F32 = torch.float32

# A workgroup that stays and walks through several tiles, its loads ahead of
# them: at each size of a tile, each pair of operands that has that many tiles.
WALK_GATED = [(SHORT, 8197, 129, 1637), ([F32], 1500, 71, 3767), ([F32], 36, 1432, 3922), ([F32], 8197, 1260, 25)]
WALK_XENT = [(SHORT, 130, 1312, 34067), (SHORT, 4305, 68, 4033), (SHORT, 3784, 138, 42168), (SHORT, 21, 443, 40688),
             ([F32], 23, 608, 17785), ([F32], 8197, 1374, 264), ([F32], 8197, 477, 8667)]

# The tiles of the gradients' products (operands read transposed, whole or in
# parts, added to an earlier piece's) at the sizes that the shapes above leave
# out; vocabularies of several pieces in each type, with a short last one.
GRADIENT_GATED = [(SHORT, 4100, 1032, 2050), (SHORT, 1500, 1368, 718), (SHORT, 4950, 1688, 2329),
                  ([F32], 2049, 1000, 1500), ([F32], 2639, 1602, 1354)]
GRADIENT_XENT = [(SHORT, 1500, 1000, 8200), (SHORT, 4100, 520, 35000), (SHORT, 4100, 264, 35000),
                 (SHORT, 6817, 69, 19772), ([F32], 1989, 70, 42247), ([F32], 2688, 1565, 219)]


def each(shapes):
    return [(t, *s) for types, *s in shapes for t in types]


@pytest.mark.parametrize("dtype,rows,width,hidden", each(WALK_GATED))
def test_gated_several_tiles_a_workgroup(ops, dtype, rows, width, hidden):  # noqa: F811
    gated_case(ops, dtype, rows, width, hidden, "silu")


@pytest.mark.parametrize("dtype,rows,width,vocab", each(WALK_XENT))
def test_softmax_xent_several_tiles_a_workgroup(ops, dtype, rows, width, vocab):  # noqa: F811
    xent_case(ops, dtype, rows, width, vocab, rows % 2 == 0)


@pytest.mark.parametrize("dtype", SHORT + [F32])
def test_several_tiles_a_workgroup_same_bits(ops, dtype):  # noqa: F811
    """What is read before it is loaded, or loaded before it is read, differs from run to run."""
    x, w = rand(1, 2300, 712, dtype=dtype), rand(2, 12000, 712, scale=0.05, dtype=dtype)
    labels = (torch.arange(2300, device="cuda") * 5).to(torch.int32)
    dloss, dh = rand(3, 2300), rand(4, 2300, 6000, dtype=dtype)

    def run():
        loss, lse = ops.softmax_xent(x, w, labels)
        out = [loss, *ops.softmax_xent_backward(dloss, lse, x, w, labels)[:2]]
        return out + [ops.gated(x, w[:6000], w[6000:]), *ops.gated_backward(dh, x, w[:6000], w[6000:])]

    first = run()
    for _ in range(4):
        for a, b in zip(first, run()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,rows,width,hidden", each(GRADIENT_GATED))
def test_gated_gradient_tiles(ops, dtype, rows, width, hidden):  # noqa: F811
    gated_case(ops, dtype, rows, width, hidden, "gelu" if hidden % 2 else "sigmoid")


@pytest.mark.parametrize("dtype,rows,width,vocab", each(GRADIENT_XENT))
def test_softmax_xent_gradient_tiles(ops, dtype, rows, width, vocab):  # noqa: F811
    xent_case(ops, dtype, rows, width, vocab, rows % 2 == 1)


@pytest.mark.parametrize("dtype", SHORT + [F32])
@pytest.mark.parametrize("width,pad,offset", [(1000, 8, 8), (1001, 3, 1)])
def test_gradient_tiles_of_strided_matrices(ops, dtype, width, pad, offset):  # noqa: F811
    gated_case(ops, dtype, 2049, width, 1503, "silu", pad, offset)
    xent_case(ops, dtype, 2049, width, 9001, True, pad, offset)
