"""The gated recurrence (include/lda_ops.h) of matrices whose last group of columns has few of them."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import TYPES, ops  # noqa: E402,F401
from test_gpu_ops_recurrence import inputs, offsets_of  # noqa: E402

pytestmark = pytest.mark.gpu

NAMES = ("h", "last", "dx", "dgate", "dstate")


def everything(ops, x, gate, off, state, dh, dlast):  # noqa: F811
    h, last, kept = ops.recurrence(x, gate, off, state)
    return dict(zip(NAMES, (h, last, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast))))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [65, 129, 130, 193])
def test_last_group_of_few_columns(ops, dtype, cols):  # noqa: F811
    """Lanes without columns beside lanes whose rows begin and end documents: states, last states and their gradients
    of every document, as they are where the group is full."""
    lengths = [1, 2, 0, 3, 30, 31, 1, 1, 0, 64, 200, 5]
    off, rows = offsets_of(lengths, 4), sum(lengths) + 9
    given = inputs(dtype, rows, 256, len(lengths), True)
    x, gate, state, dh, dlast = given
    want = everything(ops, x, gate, off, state, dh, dlast)
    got = everything(ops, x[:, :cols], gate[:, :cols], off, state[:, :cols].contiguous(), dh[:, :cols],
                     dlast[:, :cols].contiguous())
    assert all(torch.equal(got[n], want[n][:, :cols]) for n in NAMES)
