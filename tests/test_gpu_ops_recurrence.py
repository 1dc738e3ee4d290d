"""The gated recurrence (include/lda_ops.h) against its formulas in 64 bits.

Bounds, with E = 2^-24: exp(-g) is within 4 E of itself and what its argument's
rounding, |g| E and as much again, makes of it; the gate 1 / (1 + e) and one
minus it, e times the gate, take at most R = (12 + 3 |g|) E of themselves.  The
state is a sum of terms, each a product of gates, one (1 - f) and one x, in
whatever order the products and sums are taken: with M_t = f M_{t-1} + (1 - f) |x|
the sum of their magnitudes, a step adds (R + 3 E) M_t to the error that it
passes on.  The gradients run the other way in the same manner.
"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, TYPES, check, directional, ops, rand, strided, STEP, ROOM  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def offsets_of(lengths, first=0):
    return torch.tensor([first] + [first + sum(lengths[:i + 1]) for i in range(len(lengths))], dtype=torch.int64,
                        device="cuda")


def reference(x, gate, bounds, state, dh, dlast):
    """Values and bounds of everything, on the CPU, a document after another."""
    x, gate = x.cpu().to(F8), gate.cpu().to(F8)
    rows, cols = x.shape
    docs = len(bounds) - 1
    f, k = torch.sigmoid(gate), torch.sigmoid(-gate)
    r = (12 + 3 * gate.abs()) * E
    zero = torch.zeros(cols, dtype=F8)
    out = {n: torch.zeros(rows, cols, dtype=F8) for n in ("h", "dx", "dgate")}
    out.update({n: torch.zeros(docs, cols, dtype=F8) for n in ("last", "dstate")})
    bound = {n: torch.zeros_like(t) for n, t in out.items()}
    for s in range(docs):
        begin, end = bounds[s], bounds[s + 1]
        first = state[s].cpu().to(F8) if state is not None else zero
        dl = dlast[s].cpu().to(F8) if dlast is not None else zero
        if end <= begin:
            out["last"][s], out["dstate"][s] = first, dl
            continue
        h, d, m = first, zero, first.abs()
        before, dbefore, mbefore = [], [], []
        for t in range(begin, end):
            before.append(h)
            dbefore.append(d)
            mbefore.append(m)
            h = f[t] * h + k[t] * x[t]
            m = f[t] * m + k[t] * x[t].abs()
            d = f[t] * d + (r[t] + 3 * E) * m
            out["h"][t], bound["h"][t] = h, d
        out["last"][s], bound["last"][s] = h, d
        if dh is None:
            continue
        grad, d, m = dl, zero, dl.abs()
        for t in range(end - 1, begin - 1, -1):
            now = dh[t].cpu().to(F8)
            grad, m = grad + now, m + now.abs()
            d = d + 3 * E * m
            i = t - begin
            size = mbefore[i] + x[t].abs()
            out["dx"][t], bound["dx"][t] = k[t] * grad, k[t] * (d + (r[t] + 3 * E) * m)
            out["dgate"][t] = grad * (before[i] - x[t]) * f[t] * k[t]
            bound["dgate"][t] = f[t] * k[t] * (d * size + m * dbefore[i] + (2 * r[t] + 6 * E) * m * size)
            grad, d, m = f[t] * grad, f[t] * d + (r[t] + 3 * E) * f[t] * m, f[t] * m
        out["dstate"][s], bound["dstate"][s] = grad, d
    return ({n: t.cuda() for n, t in out.items()}, {n: t.cuda() for n, t in bound.items()})


def inputs(dtype, rows, cols, docs, with_state, pad=0, offset=0, level=1.0):
    x = strided(rand(1, rows, cols, dtype=dtype), pad, offset)
    gate = strided((rand(2, rows, cols) * 1.5 + level).to(dtype), pad, offset)
    state = rand(3, docs, cols) if with_state else None
    return x, gate, state, strided(rand(4, rows, cols, dtype=dtype), pad, offset), rand(5, docs, cols)


def case(ops, dtype, rows, cols, offsets, with_state, with_dlast=True, pad=0, offset=0, level=1.0):  # noqa: F811
    docs = offsets.shape[0] - 1
    x, gate, state, dh, dlast = inputs(dtype, rows, cols, docs, with_state, pad, offset, level)
    dlast = dlast if with_dlast else None
    bounds = [min(max(int(o), 0), rows) for o in offsets]
    want, bound = reference(x, gate, bounds, state, dh, dlast)
    h, last, kept = ops.recurrence(x, gate, offsets, state)
    check("h", h, want["h"], bound["h"])
    check("last", last, want["last"], bound["last"])
    dx, dgate, dstate = ops.recurrence_backward(dh, x, gate, offsets, kept, state, dlast)
    check("dx", dx, want["dx"], bound["dx"])
    check("dgate", dgate, want["dgate"], bound["dgate"])
    assert (dstate is None) == (state is None)
    if with_state:
        check("dstate", dstate, want["dstate"], bound["dstate"])
    outside = torch.ones(rows, dtype=torch.bool)
    outside[bounds[0]:bounds[-1]] = False
    for t in (h, dx, dgate):
        assert not bool(t[outside.cuda()].any())


# a wave has 16 or 32 rows, a workgroup 128 or 256; documents of one row, empty ones, ones over the ends of both
LENGTHS = [[1], [2], [31], [32], [33], [255], [256], [257], [1, 1, 1], [0, 5, 0, 0, 3, 0], [32, 32], [31, 1, 32, 1],
           [200, 300, 7, 0, 90], [256, 256, 1], [700], [1] * 70, [3] * 90 + [500], [15, 1, 16, 17], [127, 1, 128],
           [129, 127, 128, 0, 0, 128], [0] * 200 + [40] + [0] * 100 + [1, 0, 1] + [0] * 70 + [90] + [0] * 65]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", range(len(LENGTHS)))
def test_recurrence(ops, dtype, which):  # noqa: F811
    lengths = LENGTHS[which]
    cols = [1, 7, 64, 130, 65][which % 5]
    case(ops, dtype, sum(lengths), cols, offsets_of(lengths), which % 2 == 0, which % 3 != 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [2, 6, 96, 129, 256])
@pytest.mark.parametrize("pad,offset", [(3, 1), (2, 2), (8, 8), (1, 0)])
def test_recurrence_widths_and_strides(ops, dtype, cols, pad, offset):  # noqa: F811
    case(ops, dtype, 300, cols, offsets_of([100, 150, 50]), True, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 2, 3, 5001])
def test_recurrence_narrow_and_wide(ops, dtype, cols):  # noqa: F811
    case(ops, dtype, 50, cols, offsets_of([3, 47]), True)
    case(ops, dtype, 50, cols, offsets_of([50]), False, pad=1, offset=1)


def test_recurrence_far_offsets(ops):  # noqa: F811
    """Elements beyond 2^32 of their matrices: the last documents as they are by themselves."""
    rows, cols = 4300000, 1024
    tail = 3000
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    gate = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda").expand(rows, cols)
    x[-tail:] = rand(1, tail, cols, dtype=torch.bfloat16)
    off = torch.tensor([0, rows - tail, rows - tail + 1000, rows], device="cuda")
    h, last, kept = ops.recurrence(x, gate, off)
    alone, alone_last, alone_kept = ops.recurrence(x[-tail:], gate[:tail], off[1:] - off[1])
    assert not bool(h[:-tail].any())
    # one rounding to bf16, on either side of a border, of states that are some 100 roundings of 32 bits apart
    assert bool(((h[-tail:] - alone).float().abs() <= 2 * 2.0 ** -8 * alone.float().abs() + 1e-5).all())
    assert torch.allclose(last[1:], alone_last, rtol=0, atol=1e-4 * float(alone_last.abs().max()))
    dx, dgate, _ = ops.recurrence_backward(x, x, gate, off, kept)
    adx, adgate, _ = ops.recurrence_backward(x[-tail:], x[-tail:], gate[:tail], off[1:] - off[1], alone_kept)
    for a, b in ((dx, adx), (dgate, adgate)):
        assert not bool(a[:-tail].any())
        assert bool(((a[-tail:] - b).float().abs() <= 2 * 2.0 ** -8 * b.float().abs() + 1e-4).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_rows_of_no_document(ops, dtype):  # noqa: F811
    """Rows before the first document and behind the last one, and offsets that lie outside the rows."""
    case(ops, dtype, 400, 40, offsets_of([60, 0, 200], 50), True)
    case(ops, dtype, 90, 40, offsets_of([30], 60), False)
    case(ops, dtype, 300, 10, torch.tensor([-70, -5, 100, 420, 500], device="cuda"), True)
    case(ops, dtype, 300, 10, torch.tensor([0], device="cuda"), False)
    case(ops, dtype, 20, 10, torch.tensor([0, 0, 0], device="cuda"), True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("level", [-2.0, 4.0])
def test_recurrence_long_document(ops, dtype, level):  # noqa: F811
    """More workgroups than one look back takes in, with gates that keep and gates that forget."""
    case(ops, dtype, 10300, 70, offsets_of([40, 10200, 0, 60]), True, level=level)


def test_recurrence_far_gates(ops):  # noqa: F811
    """Gates of 0 and 1: the row itself, or the state before it; no infinity on the way."""
    rows, cols = 70, 6
    x, state = rand(1, rows, cols), rand(2, 1, cols)
    off = offsets_of([rows])
    dh, dlast = torch.zeros(rows, cols, device="cuda"), torch.ones(1, cols, device="cuda")
    for big in (100.0, 3e38, float("inf")):
        gate = torch.full((rows, cols), big, device="cuda")
        h, last, kept = ops.recurrence(x, gate, off, state)
        assert torch.equal(h, state.expand(rows, cols)) and torch.equal(last, state)
        dx, dgate, dstate = ops.recurrence_backward(dh, x, gate, off, kept, state, dlast)
        assert bool((dx.abs() <= 1e-30).all()) and bool((dgate.abs() <= 1e-30).all())
        assert torch.equal(dstate, dlast)
        h, last, kept = ops.recurrence(x, -gate, off, state)
        assert torch.equal(h, x) and torch.equal(last, x[-1:])
        dx, dgate, dstate = ops.recurrence_backward(dh, x, -gate, off, kept, state, dlast)
        assert torch.equal(dx[-1:], dlast) and not bool(dx[:-1].abs().gt(1e-30).any())
        assert bool((dgate.abs() <= 1e-30).all()) and bool((dstate.abs() <= 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_recurrence_bad_values_stay_in_their_document(ops, dtype, bad):  # noqa: F811
    """Infinities and NaN in a document and in padding leave every other document's bits as they are."""
    lengths = [40, 300, 5, 600, 20, 1]
    rows, cols = sum(lengths) + 33, 66
    off = offsets_of(lengths, 13)
    x, gate, state, dh, dlast = inputs(dtype, rows, cols, len(lengths), True)

    def everything():
        h, last, kept = ops.recurrence(x, gate, off, state)
        return [h, last, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast)]

    want = [t.clone() for t in everything()]
    row = torch.arange(rows, device="cuda")
    hurt = (row < 13) | (row >= 13 + sum(lengths)) | ((row >= 53) & (row < 353)) | ((row >= 358) & (row < 958))
    x[60], gate[70], dh[80] = bad, bad, bad
    x[500], gate[400, 5], dh[900] = bad, -bad, bad
    state[1], dlast[3] = bad, bad
    for t in (x, gate, dh):
        t[:13], t[13 + sum(lengths):] = bad, bad
    got = everything()
    docs = torch.tensor([0, 2, 4, 5], device="cuda")
    for name, a, b in zip(("h", "last", "dx", "dgate", "dstate"), got, want):
        sound = docs if name in ("last", "dstate") else torch.nonzero(~hurt)[:, 0]
        assert torch.equal(a[sound], b[sound]), name
    pad = (row < 13) | (row >= 13 + sum(lengths))
    for t in (got[0], got[2], got[3]):
        assert not bool(t[pad].any())
    assert not bool(got[0][60:70].isfinite().any())


def test_recurrence_empty(ops):  # noqa: F811
    x = torch.empty(0, 24, device="cuda")
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    state, dlast = rand(1, 3, 24), rand(2, 3, 24)
    h, last, kept = ops.recurrence(x, x, off, state)
    assert h.shape == (0, 24) and torch.equal(last, state) and kept.shape == (0, 24)
    assert not bool(ops.recurrence(x, x, off)[1].any())
    dx, dgate, dstate = ops.recurrence_backward(x, x, x, off, kept, state, dlast)
    assert dx.shape == dgate.shape == (0, 24) and torch.equal(dstate, dlast)
    h, last, _ = ops.recurrence(x, x, off[:1])
    assert last.shape == (0, 24)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1024), (5, 7), (64, 130), (300, 1000)])
def test_recurrence_step(ops, dtype, rows, cols):  # noqa: F811
    """One row more, against the formula and, word after word, against the whole document at once."""
    for pad, offset in ((0, 0), (3, 1)):
        x, gate, state, _, _ = inputs(dtype, rows, cols, rows, True, pad, offset)
        h, new = ops.recurrence_step(x, gate, state)
        want, bound = reference(x, gate, list(range(rows + 1)), state, None, None)
        check("h", h, want["h"], bound["h"])
        check("state", new, want["last"], bound["last"])
        assert not torch.equal(new, state)
        again = state.clone()
        h2, new2 = ops.recurrence_step(x, gate, again, out=again)
        assert new2 is again and torch.equal(again, new) and torch.equal(h, h2)


def test_recurrence_steps_follow_the_documents(ops):  # noqa: F811
    """Words of three documents one at a time, from the state that a first part left: the whole at once."""
    cols, length = 70, 50
    x, gate = rand(1, 3 * length, cols), rand(2, 3 * length, cols) + 1
    whole, last, _ = ops.recurrence(x, gate, offsets_of([length] * 3))
    head = torch.cat([torch.arange(20) + i * length for i in range(3)]).cuda()
    _, state, _ = ops.recurrence(x[head], gate[head], offsets_of([20] * 3))
    # terms of at most max |x|, 50 rows that add R + 3 E of it each, twice
    room = 4 * length * 30 * E * float(x.abs().max())
    for t in range(20, length):
        at = torch.arange(3, device="cuda") * length + t
        h, _ = ops.recurrence_step(x[at], gate[at], state, out=state)
        assert bool(((h - whole[at]).abs() <= room).all())
    assert bool(((state - last).abs() <= room).all())


def test_recurrence_gradients_against_differences(ops):  # noqa: F811
    off = offsets_of([30, 0, 45, 5])
    x, gate, state = rand(1, 80, 20), rand(2, 80, 20), rand(3, 4, 20)
    c, cl = rand(4, 80, 20), rand(5, 4, 20)

    def value(t):
        h, last, _ = ops.recurrence(t[0], t[1], off, t[2])
        return float((h.to(F8) * c.to(F8)).sum() + (last.to(F8) * cl.to(F8)).sum())

    _, _, kept = ops.recurrence(x, gate, off, state)
    grads = ops.recurrence_backward(c, x, gate, off, kept, state, cl)
    got, want = directional(value, grads, [x, gate, state], 10, STEP)
    assert abs(got - want) <= ROOM * max(1.0, abs(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_recurrence_bad_documents_between_sound_ones(ops, dtype, bad):  # noqa: F811
    """Documents of nothing but infinities or NaN, which begin and end inside the rows of a wave."""
    lengths = [5, 7, 200, 20, 3, 1, 400, 300, 90]
    rows, cols = sum(lengths), 10
    off = offsets_of(lengths)
    x, gate, state, dh, dlast = inputs(dtype, rows, cols, len(lengths), True)

    def everything():
        h, last, kept = ops.recurrence(x, gate, off, state)
        return [h, last, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast)]

    want = [t.clone() for t in everything()]
    sound = torch.ones(rows, dtype=torch.bool, device="cuda")
    for s in (1, 3, 5, 7):
        part = slice(int(off[s]), int(off[s + 1]))
        sound[part] = False
        for t in (x, gate, dh):
            t[part] = bad
        state[s], dlast[s] = bad, bad
    got = everything()
    for name, a, b in zip(("h", "last", "dx", "dgate", "dstate"), got, want):
        at = slice(0, None, 2) if name in ("last", "dstate") else sound
        assert torch.equal(a[at], b[at]), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [129, 257, 385])
def test_recurrence_columns_of_two_workgroups(ops, dtype, cols):  # noqa: F811
    """A row's last column alone in a part of 128, so that its pair has a column of the part before: the bits that it
    has with a column after it, which makes the pair whole."""
    rows = 30000
    off = offsets_of([rows - 900, 900])
    x, gate, state, dh, dlast = inputs(dtype, rows, cols + 1, 2, True, level=4.0)

    def everything(n):
        first = state[:, :n].contiguous()
        h, last, kept = ops.recurrence(x[:, :n], gate[:, :n], off, first)
        return [h, last, kept, *ops.recurrence_backward(dh[:, :n], x[:, :n], gate[:, :n], off, kept, first,
                                                        dlast[:, :n].contiguous())]

    want = everything(cols + 1)
    for _ in range(5):
        for a, b in zip(everything(cols), want):
            assert torch.equal(a, b[:, :cols])


def test_recurrence_same_bits_and_streams(ops):  # noqa: F811
    """Long and short documents: the same bits whichever workgroup comes first, on any stream, twice at once."""
    lengths = [9000, 3, 0, 500, 20000, 100]
    rows = sum(lengths)
    off = offsets_of(lengths)
    x, gate, state, dh, dlast = inputs(torch.bfloat16, rows, 136, len(lengths), True, level=3.0)

    def everything():
        h, last, kept = ops.recurrence(x, gate, off, state)
        return [h, last, kept, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast)]

    want = everything()
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(everything())
    torch.cuda.synchronize()
    for one in got:
        for a, b in zip(want, one):
            assert torch.equal(a, b)


def test_recurrence_in_a_graph(ops):  # noqa: F811
    """Captured once, replayed on new contents, with the program's own work between."""
    off = offsets_of([300, 0, 1000, 40])
    x, gate, state, dh, dlast = inputs(torch.float32, 1400, 66, 4, True)

    def everything():
        h, last, kept = ops.recurrence(x, gate, off, state)
        return [h, last, *ops.recurrence_backward(dh, x, gate, off, kept, state, dlast)]

    everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for i in range(4):
        x.copy_(rand(20 + i, 1400, 66))
        off[1:3] = 200 + 50 * i
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, everything()):
            assert torch.equal(a, b), i


def test_recurrence_joint_matrix_and_broadcast(ops):  # noqa: F811
    """x and gate as halves of one matrix; one row in memory for all."""
    both = rand(1, 500, 144, dtype=torch.bfloat16)
    off = offsets_of([250, 250])
    a = ops.recurrence(both[:, :72], both[:, 72:], off)
    b = ops.recurrence(both[:, :72].contiguous(), both[:, 72:].contiguous(), off)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    one = both[:1, :72].expand(500, 72)
    a = ops.recurrence(one, one, off)
    b = ops.recurrence(one.contiguous(), one.contiguous(), off)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_recurrence_refusals(ops):  # noqa: F811
    x, gate, state, dh, dlast = inputs(torch.float32, 10, 8, 2, True)
    off, two = offsets_of([4, 6]), rand(6, 3, 8)
    _, _, kept = ops.recurrence(x, gate, off, state)
    bad = [lambda: ops.recurrence(x.cpu(), gate, off), lambda: ops.recurrence(x, gate[:5], off),
           lambda: ops.recurrence(x, gate.half(), off), lambda: ops.recurrence(x, gate, off.int()),
           lambda: ops.recurrence(x, gate, off.cpu()), lambda: ops.recurrence(x, gate, off[:0]),
           lambda: ops.recurrence(x, gate, off, state[:1]), lambda: ops.recurrence(x, gate, off, state.half()),
           lambda: ops.recurrence(x, gate, off, state[:, :4].expand(2, 4)), lambda: ops.recurrence(x.t(), gate.t(), off),
           lambda: ops.recurrence(x, gate, off, rand(1, 2, 9)[:, :8]),
           lambda: ops.recurrence(x, gate, None), lambda: ops.recurrence(x, gate, off[::2]),
           lambda: ops.recurrence(x.clone().requires_grad_(), gate, off),
           lambda: ops.recurrence_backward(dh[:5], x, gate, off, kept, state, dlast),
           lambda: ops.recurrence_backward(dh, x, gate, off, kept[:0], state, dlast),
           lambda: ops.recurrence_backward(dh, x, gate, off, kept.half(), state, dlast),
           lambda: ops.recurrence_backward(dh, x, gate, off, kept, state, dlast[:1]),
           lambda: ops.recurrence_step(x, gate, state), lambda: ops.recurrence_step(x[:2], gate[:2], state.half()),
           lambda: ops.recurrence_step(x[:2], gate[:2], state, out=state[:1]),
           lambda: ops.recurrence_step(x[:2], gate[:2], state, out=state.double()),
           lambda: ops.recurrence_step(x[:2], gate[:2], two[:2], out=two[1:])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d did not come" % i)
