"""Word-model operators where a type's range or precision is what decides, against their formulas in 64 bits.

Bounds are elementwise and made as in test_gpu_ops.py (u the unit roundoff of
the matrices' type, e = 2^-24, g(n) = (n + 8) e).  What a 16-bit operand adds
below its type's normal numbers is stated with each test.
"""
import math

import pytest

from test_gpu_ops import E, F8, U, check, g, gate, ops, rand  # noqa: F401 (ops is a fixture)

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

F16 = torch.float16


def telling(name, ref, bound, dtype):
    """The bound is small beside the values: a result of zeros or of infinities does not pass."""
    assert float(ref.abs().max()) < torch.finfo(dtype).max, name
    assert float((2 * bound).median()) < 0.1 * float(ref.abs().median()), name


# ------------------------------------------------------------ gated layer ---
# (scales of dh, x, w_gate and w_value, the outputs that half precision holds at
# them).  x times w_gate is of order 1 throughout.  First da and db are below
# 2^-14, then past 65,504.
SCALES = [(1e-5, 1 / 300, 300.0, 3.0, ("dx",)), (1e-5, 100.0, 0.01, 1e-4, ("dw_gate", "dw_value")),
          (2000.0, 30.0, 1 / 30, 1.5, ("dx",)), (2000.0, 1 / 300, 300.0, 12000.0, ("dw_gate", "dw_value"))]


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("rows,width,hidden", [(200, 64, 96), (70, 33, 41)])
@pytest.mark.parametrize("unequal", [False, True])
@pytest.mark.parametrize("scales", SCALES)
def test_gated_half_precision_gradients_of_any_size(ops, act, rows, width, hidden, unequal, scales):  # noqa: F811
    """da and db in half precision: no infinity and no lost bits where the gradients hold.

    A row of da and db is kept times a power of two that brings B = max |dh|
    (1.2 |x| |w| + 1), which bounds it, to 2^14 at least: an entry is off by half
    a step of the subnormal numbers, 2^-25 / (2^14 / B) = B 2^-39, beside u of
    itself.  x is kept times a power of two for all rows that brings the largest
    X B (X the row's largest |x|) to the same size, and a row's entry is off by
    2^-39 max(X B) / B.
    """
    dh_scale, x_scale, gate_scale, value_scale, outputs = scales
    x = rand(1, rows, width, scale=x_scale, dtype=F16)
    wg = rand(2, hidden, width, scale=gate_scale * width ** -0.5, dtype=F16)
    wv = rand(3, hidden, width, scale=value_scale * width ** -0.5, dtype=F16)
    dh = rand(4, rows, hidden, scale=dh_scale)
    if unequal:  # rows of a 1,024th of the others
        dh[::3] *= 2.0 ** -10 if dh_scale > 1 else 2.0 ** 10
    dh = dh.to(F16)
    got = dict(zip(("dx", "dw_gate", "dw_value"), ops.gated_backward(dh, x, wg, wv, act)))
    x8, g8, v8, d8 = (t.to(F8) for t in (x, wg, wv, dh))
    a, b = x8 @ g8.t(), x8 @ v8.t()
    ea, eb = g(width) * (x8.abs() @ g8.abs().t()), g(width) * (x8.abs() @ v8.abs().t())
    p, dp = gate(act, a)
    ep, edp = 1.2 * ea + 8 * E * (p.abs() + a.abs()), ea + 8 * E * (1 + a.abs())
    da, db = d8 * b * dp, d8 * p
    longest = max(float(g8.norm(dim=1).max()), float(v8.norm(dim=1).max()))
    B = d8.abs().amax(1) * (1.2 * x8.norm(dim=1) * longest + 1)
    XB = float((x8.abs().amax(1) * B).max())
    u = U[F16] + 3 * E
    low = (B * 2.0 ** -39)[:, None]
    eda = d8.abs() * (eb * dp.abs() + b.abs() * edp) + u * da.abs() + low
    edb = d8.abs() * ep + u * db.abs() + low
    ones = torch.full_like(x8, 2.0 ** -39 * XB) / B[:, None]
    refs = dict(dx=da @ g8 + db @ v8, dw_gate=da.t() @ x8, dw_value=db.t() @ x8)
    bounds = dict(dx=(eda + g(2 * hidden) * da.abs()) @ g8.abs() + (edb + g(2 * hidden) * db.abs()) @ v8.abs(),
                  dw_gate=(eda + g(rows) * da.abs()).t() @ x8.abs() + da.abs().t() @ ones,
                  dw_value=(edb + g(rows) * db.abs()).t() @ x8.abs() + db.abs().t() @ ones)
    for name in outputs:
        telling(name, refs[name], bounds[name], F16)
        check(name, got[name], refs[name], bounds[name])


@pytest.mark.parametrize("scales", SCALES)
def test_gated_half_precision_gradients_of_many_rows(ops, scales):  # noqa: F811
    """More rows than one workgroup finds the scales of."""
    test_gated_half_precision_gradients_of_any_size(ops, "silu", 2500, 40, 72, True, scales)


def test_gated_half_precision_rows_without_gradient(ops):  # noqa: F811
    """A row whose gradient is 0 takes no part, whatever its size, and one with NaN stays in its row of dx."""
    rows, width, hidden = 40, 48, 24
    x, dh = rand(1, rows, width, dtype=F16), rand(2, rows, hidden, dtype=F16)
    wg, wv = rand(3, hidden, width, scale=0.1, dtype=F16), rand(4, hidden, width, scale=0.1, dtype=F16)
    x[5], dh[5] = 3e4, 0.0
    got = ops.gated_backward(dh, x, wg, wv)
    keep = [i for i in range(rows) if i != 5]
    want = ops.gated_backward(dh[keep].contiguous(), x[keep].contiguous(), wg, wv)
    assert torch.equal(got[0][keep], want[0]) and not bool(got[0][5].any())
    # the sum over rows has another order
    for a, b in zip(got[1:], want[1:]):
        assert bool(a.isfinite().all())
        bound = (2 * U[F16] + 2 * g(rows)) * (rows * float(x[keep].abs().max()) * float(dh.abs().max()))
        assert float((a.to(F8) - b.to(F8)).abs().max()) <= bound
    nothing = ops.gated_backward(torch.zeros_like(dh), x, wg, wv)
    assert not any(bool(t.any()) for t in nothing)
    x[7, 3] = float("nan")
    dx = ops.gated_backward(dh, x, wg, wv)[0]
    assert bool(dx[7].isnan().all()) and torch.equal(dx[[i for i in keep if i != 7]], got[0][[i for i in keep if i != 7]])


@pytest.mark.parametrize("rows", [13, 4001])
def test_gelu_in_single_precision(ops, rows):  # noqa: F811
    """gelu and its derivative relative to themselves, on both sides of 0.

    Phi(a) = erfc(-a / sqrt 2) / 2: the argument is off by 2 e of itself, which
    changes Phi by up to a^2 + 1 times that; erfc by 8 e of itself.  The bell
    exp(-a^2 / 2) is off by a^2 e, and 6 e of itself.
    """
    x = torch.linspace(-6, 6, rows, device="cuda")[:, None].contiguous()
    one = torch.ones(1, 1, device="cuda")
    a = x.to(F8)
    p, dp = gate("gelu", a)
    phi, bell = torch.special.ndtr(a), a.abs() * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    rel = (2 * (a * a + 1) + 8) * E
    check("h", ops.gated(x, one, one, "gelu"), p * a, (rel + 2 * E) * (p * a).abs())
    dx, _, _ = ops.gated_backward(torch.ones_like(x), x, one, one, "gelu")
    edp = rel * phi + (a * a + 6) * E * bell
    check("dx", dx, a * dp + p, a.abs() * edp + (rel + 4 * E) * p.abs() + 4 * E * (a * dp).abs())


# ---------------------------------------------------- softmax cross entropy ---
def xent_gradients(ops, x, w, labels, bias, dloss):  # noqa: F811
    """The operator's dx and dweight, the formulas' in 64 bits, and bounds on what is off.

    G = p - [label] is off by the logits' errors times p, by its rounding u, and
    in half precision, where it is kept times 2^14, by half a step of the
    subnormal numbers, 2^-39.  x dloss is off by its rounding u, and by 2^-39 of
    the largest, which is kept at 2^14 at least.
    """
    dtype, rows, width, vocab = x.dtype, x.shape[0], x.shape[1], w.shape[0]
    _, lse = ops.softmax_xent(x, w, labels, bias)
    dx, dw, _ = ops.softmax_xent_backward(dloss, lse, x, w, labels, bias)
    x8, w8, d8 = x.to(F8), w.to(F8), dloss.to(F8)[:, None]
    z, mag = x8 @ w8.t(), x8.abs() @ w8.abs().t()
    if bias is not None:
        z, mag = z + bias.to(F8), mag + bias.to(F8).abs()
    top = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - top)
    # a logit's error, that of the lse (the largest logit's, the sum's, its own
    # rounding), and of the exponential's argument, of at most 64 where p is not 0
    ez = g(width) * mag
    ep = p * (2 * (ez + ez.amax(1, keepdim=True) + g(vocab) + 2 * E * top.abs()) + 8 * E * 64)
    grad = p.clone()
    grad[torch.arange(rows, device="cuda"), labels.long()] -= 1
    u = (U[dtype] if dtype != torch.float32 else 0.0) + 4 * E
    eg = ep + u * grad.abs() + 2.0 ** -39
    xd = (x8 * d8).abs()
    exd = u * xd + 2.0 ** -39 * xd.max()
    refs = ((grad * d8) @ w8, (grad * d8).t() @ x8)
    bounds = (((eg + g(vocab) * grad.abs()) * d8.abs()) @ w8.abs(),
              (eg + g(rows) * grad.abs()).t() @ xd + grad.abs().t() @ exd)
    return dict(dx=(dx, refs[0], bounds[0]), dweight=(dw, refs[1], bounds[1]))


@pytest.mark.parametrize("rows,width,vocab", [(12, 64, 200), (96, 40, 400)])
@pytest.mark.parametrize("below", [8, 14, 20, 24])
def test_softmax_xent_half_precision_rows_of_unlike_gradients(ops, rows, width, vocab, below):  # noqa: F811
    """Rows whose gradient is 2^-below of the largest, with words of their own: their part of dweight keeps its bits."""
    x, w = rand(1, rows, width, dtype=F16), rand(2, vocab, width, scale=0.3 * width ** -0.5, dtype=F16)
    small = torch.arange(rows, device="cuda") % 2 == 1
    # the small rows' words are all but impossible for the others
    labels = torch.arange(rows, dtype=torch.int32, device="cuda")
    bias = rand(3, vocab)
    bias[:rows][small] = -40.0
    dloss = torch.full((rows,), 2.0 ** 12, device="cuda")
    dloss[small] = torch.linspace(1.0, 1.9, int(small.sum()), device="cuda") * 2.0 ** (12 - below)
    got, ref, bound = xent_gradients(ops, x, w, labels, bias, dloss)["dweight"]
    telling("dweight", ref[:rows], bound[:rows], F16)
    check("dweight", got, ref, bound)


@pytest.mark.parametrize("x_scale,w_scale,name", [(2e4, 1e-4, "dweight"), (1e-4, 2e4, "dx")])
@pytest.mark.parametrize("dloss_scale", [2.0 ** -26, 2.0 ** -20])
@pytest.mark.parametrize("rows", [12, 200])
def test_softmax_xent_half_precision_small_gradients(ops, x_scale, w_scale, name, dloss_scale, rows):  # noqa: F811
    """Gradients far below half precision's range, of results that are in it."""
    x, w = rand(1, rows, 64, scale=0.5 * x_scale, dtype=F16), rand(2, 300, 64, scale=w_scale / 8, dtype=F16)
    if name == "dx":
        w = rand(2, 300, 64, scale=0.5 * w_scale, dtype=F16)
        x = rand(1, rows, 64, scale=x_scale / 8, dtype=F16)
    labels = (torch.arange(rows, device="cuda") * 7 % 300).to(torch.int32)
    got, ref, bound = xent_gradients(ops, x, w, labels, None, rand(4, rows, scale=dloss_scale))[name]
    shown = ref[labels.long().unique()] if name == "dweight" else ref
    telling(name, shown, bound[labels.long().unique()] if name == "dweight" else bound, F16)
    check(name, got, ref, bound)
