"""Word-model operators on tensors that require a gradient: torch gets none from them, so they refuse."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def calls():
    from paper_2007_08725_amd import ops
    x, w = torch.randn(4, 16, device="cuda"), torch.randn(8, 16, device="cuda")
    v, u, dh, rows = (torch.randn(n, device="cuda") for n in ((16,), (8,), (4, 8), (4,)))
    labels = torch.zeros(4, dtype=torch.int32, device="cuda")
    return [(ops.layer_norm, [x, v, v.clone()]), (ops.layer_norm_backward, [x, x.clone(), v, rows, rows.clone()]),
            (ops.gated, [x, w, w.clone()]), (ops.gated_backward, [dh, x, w, w.clone()]),
            (ops.softmax_xent, [x, w, labels, u]),
            (ops.softmax_xent_backward, [rows, rows.clone(), x, w, labels, u])]


@pytest.mark.parametrize("which", range(6))
def test_tensors_that_require_a_gradient_are_refused(which):
    call, args = calls()[which]
    want = call(*args)
    for i, t in enumerate(args):
        if not t.is_floating_point():
            continue
        given = list(args)
        given[i] = t.clone().requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            call(*given)
        with torch.no_grad():
            got = call(*given)
        given[i] = given[i].detach()
        for a, b, c in zip(*(r if isinstance(r, tuple) else (r,) for r in (want, got, call(*given)))):
            assert torch.equal(a, b) and torch.equal(a, c)
