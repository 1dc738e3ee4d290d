"""Distillation of as many rows as a call takes: a workgroup of 256 a row is 2^32 threads, more than one launch has."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import E, F8, g, ops, rand  # noqa: E402,F401
from test_gpu_ops_many_rows import room_for, rows_are  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_softmax_distill(ops, dtype):  # noqa: F811
    """All rows are one row in memory, so every output row is the same; the last one comes from a second launch."""
    rows, width, vocab, top = ops.MAX_ROWS, 8, 100, 2
    room_for(rows * (vocab + 4) * 8)
    x, w = rand(1, 1, width, dtype=dtype), rand(2, vocab, width, dtype=dtype)
    words = torch.tensor([[7, 99]], dtype=torch.int32, device="cuda")
    scores = torch.tensor([[-1.0, -2.5]], device="cuda")
    given = (x.expand(rows, width), w, words.expand(rows, top), scores.expand(rows, top))
    loss, lse, logits = ops.softmax_distill(*given)
    z, mag = (x.to(F8) @ w.to(F8).t())[0], (x.to(F8).abs() @ w.to(F8).abs().t())[0]
    p = torch.softmax(scores.to(F8)[0], 0)
    listed, total = z[words[0].long()], torch.logsumexp(z, 0)
    want = (p * (torch.log(p) - listed + total)).sum()
    # a logit is off by its sum's roundings, the lse by the largest logit's, its own sum's and its last few
    off = g(width + 4) * float(mag.max())
    assert bool(((logits[-1].to(F8) - listed).abs() <= 2 * off).all())
    room = 2 * (2 * off + g(vocab) + 16 * E * (1 + float(z.abs().max()) + float(total)))
    assert abs(float(lse[-1]) - float(total)) <= room and abs(float(loss[-1]) - float(want)) <= 2 * room
    assert rows_are(logits, logits[:1]) and bool((loss == loss[0]).all()) and bool((lse == lse[0]).all())
    dloss = torch.ones(1, device="cuda").expand(rows).contiguous()
    dx, dw, _ = ops.softmax_distill_backward(dloss, lse, logits, *given)
    assert rows_are(dx, dx[:1]) and bool(dx[0].isfinite().all()) and bool(dw.isfinite().all())
    del dx, logits
    torch.cuda.empty_cache()
