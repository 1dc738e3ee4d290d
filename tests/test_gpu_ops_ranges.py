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
