"""The gated recurrence of narrow matrices (include/lda_ops.h), whose waves hold several parts of rows, over more rows
than one look back takes in: up to 64 columns of 16 bits or 32 of single precision, 256 or 512 rows to a workgroup, 32
workgroups to a look.  And of matrices whose last group of columns has few of them.

A column depends on no other, so that one reference of the widest matrix serves all; its bounds are those of
test_gpu_ops_recurrence.py.
"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, TYPES, U, check, ops, rand  # noqa: E402,F401
from test_gpu_ops_recurrence import inputs, offsets_of, reference  # noqa: E402

pytestmark = pytest.mark.gpu

WIDEST = 66
LENGTHS = [37, 12500, 0, 5000, 1, 1300, 16]
NAMES = ("h", "last", "dx", "dgate", "dstate")
_known = {}


def widest(dtype):
    """Inputs, values and bounds of all columns, made once a type (rows before and after the documents belong to none)."""
    if dtype not in _known:
        rows, docs = sum(LENGTHS) + 20, len(LENGTHS)
        off = offsets_of(LENGTHS, 9)
        x, gate, state, dh, dlast = inputs(dtype, rows, WIDEST, docs, True, level=2.0)
        host = [t.cpu() for t in (x, gate, state, dh, dlast)]
        want, bound = reference(host[0], host[1], off.tolist(), host[2], host[3], host[4])
        _known[dtype] = (x, gate, off, state, dh, dlast, want, bound)
    return _known[dtype]


def everything(ops, x, gate, off, state, dh, dlast):  # noqa: F811
    h, last, kept = ops.recurrence(x, gate, off, state)
    return dict(zip(NAMES, (h, last, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast))))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 2, 5, 16, 17, 20, 31, 32, 33, 63, 64, 65, 66])
def test_long_documents(ops, dtype, cols):  # noqa: F811
    x, gate, off, state, dh, dlast, want, bound = widest(dtype)
    first = (WIDEST - cols) // 2  # columns from the middle, at any address
    part = slice(first, first + cols)
    got = everything(ops, x[:, part], gate[:, part], off, state[:, part].contiguous(), dh[:, part],
                     dlast[:, part].contiguous())
    for name in NAMES:
        check("%s of %d columns" % (name, cols), got[name], want[name][:, part], bound[name][:, part])
    whole = everything(ops, *(t[:, part].contiguous() for t in (x, gate)), off, state[:, part].contiguous(),
                       *(t[:, part].contiguous() for t in (dh, dlast)))
    assert all(torch.equal(got[n], whole[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [1, 2, 20, 40])
def test_narrow_as_wide(ops, dtype, cols):  # noqa: F811
    """Columns by themselves against the same ones in a matrix of 200, over 30,000 rows.

    With gates of at most 2, f <= s = 0.881, errors that rows add pass on to a sum of at most 1 / (1 - s) of one row's:
    (R + 3 E) max |x| with R = (12 + 3 |g|) E for the state (test_gpu_ops_recurrence.py), twice that of the largest
    gradient, max |dh| / (1 - s), for the gradients.  Both calls may be so far off, and are rounded by half a step.
    """
    rows, width = 30000, 200
    off = offsets_of([29000, 0, 1000])
    x, gate, state, dh, dlast = inputs(dtype, rows, width, 3, True)
    gate = gate.clamp(-2, 2)
    wide = everything(ops, x, gate, off, state, dh, dlast)
    narrow = everything(ops, x[:, :cols], gate[:, :cols], off, state[:, :cols].contiguous(), dh[:, :cols],
                        dlast[:, :cols].contiguous())
    pass_on, r = 1 / (1 - 0.881), (12 + 3 * 2) * E + 3 * E
    high = max(float(x.abs().max()), float(state.abs().max()))
    steepest = max(float(dh.abs().max()), float(dlast.abs().max())) * pass_on
    room = dict(h=r * high * pass_on, last=r * high * pass_on, dx=3 * r * steepest * pass_on,
                dstate=3 * r * steepest * pass_on, dgate=3 * r * steepest * 2 * high * pass_on)
    for name in NAMES:
        a, b = narrow[name].to(F8), wide[name][:, :cols].to(F8)
        assert bool(((a - b).abs() <= 2 * room[name] + 2 * U[narrow[name].dtype] * b.abs()).all()), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 5, 20, 33, 64])
def test_same_bits_and_streams(ops, dtype, cols):  # noqa: F811
    """The same bits whichever workgroup comes first, on any stream, several at once."""
    lengths = [9000, 3, 0, 500, 20000, 100]
    off = offsets_of(lengths)
    given = inputs(dtype, sum(lengths), cols, len(lengths), True, level=3.0)
    x, gate, state, dh, dlast = given
    want = everything(ops, x, gate, off, state, dh, dlast)
    got = []
    for s in [torch.cuda.Stream() for _ in range(3)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(everything(ops, x, gate, off, state, dh, dlast))
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(one[n], want[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 5, 20, 40])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_bad_documents_between_sound_ones(ops, dtype, cols, bad):  # noqa: F811
    """Documents of nothing but infinities or NaN, which begin and end inside the rows of a part, a wave and a workgroup,
    and padding that holds the same, leave every other document's bits as they are."""
    lengths = [3, 5, 40, 20, 3, 1, 700, 300, 9000, 1, 90, 2, 5000, 77]
    off, rows = offsets_of(lengths, 11), sum(lengths) + 30
    x, gate, state, dh, dlast = inputs(dtype, rows, cols, len(lengths), True)
    want = everything(ops, x, gate, off, state, dh, dlast)
    sound = torch.ones(rows, dtype=torch.bool, device="cuda")
    for s in range(1, len(lengths), 2):
        part = slice(int(off[s]), int(off[s + 1]))
        sound[part] = False
        for t in (x, gate, dh):
            t[part] = bad
        state[s], dlast[s] = bad, bad
    for t in (x, gate, dh):
        t[:11], t[int(off[-1]):] = bad, bad
    got = everything(ops, x, gate, off, state, dh, dlast)
    for name in NAMES:
        at = slice(0, None, 2) if name in ("last", "dstate") else sound
        assert torch.equal(got[name][at], want[name][at]), name


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 20), (torch.float32, 12), (torch.bfloat16, 20),
                                        (torch.float16, 48), (torch.bfloat16, 1)])
def test_in_a_graph(ops, dtype, cols):  # noqa: F811
    """Captured once, replayed on new contents and documents, with the program's own work between."""
    rows = 19000
    off = offsets_of([300, 0, 18000, 700])
    x, gate, state, dh, dlast = inputs(dtype, rows, cols, 4, True)
    everything(ops, x, gate, off, state, dh, dlast)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything(ops, x, gate, off, state, dh, dlast)
    for i in range(4):
        x.copy_(rand(20 + i, rows, cols))
        off[1:3] = 200 + 5000 * i
        graph.replay()
        torch.cuda.synchronize()
        now = everything(ops, x, gate, off, state, dh, dlast)
        assert all(torch.equal(out[n], now[n]) for n in NAMES), i


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
