"""Layer norm of more rows than one launch has workgroups for (2^32 threads: 4,194,303 rows of 1,024 lanes)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROWS = 4194304 + 3


def room_for(count):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < count + (16 << 30):
        pytest.skip("needs %d GB of device memory" % (count >> 30))


def rows_are(m, row):
    return all(bool((m[i:i + (1 << 16)] == row).all()) for i in range(0, m.shape[0], 1 << 16))


def test_layer_norm():
    """All rows are one row in memory; 8,200 columns of half precision take 1,024 lanes."""
    from paper_2007_08725_amd import ops
    cols = 8200
    room_for(ROWS * cols * 2)
    one = torch.randn(1, cols, device="cuda", dtype=torch.float16)
    want, mean, rstd = ops.layer_norm(one)
    y, means, rstds = ops.layer_norm(one.expand(ROWS, cols))
    assert rows_are(y, want) and bool((means == mean).all()) and bool((rstds == rstd).all())
    del y
    torch.cuda.empty_cache()


def test_layer_norm_backward():
    """16,392 columns take the backward pass in two kernels, the first with 1,024 lanes a row."""
    from paper_2007_08725_amd import ops
    cols = 16392
    room_for(ROWS * cols * 2)
    one, dy = torch.randn(1, cols, device="cuda").half(), torch.randn(1, cols, device="cuda").half()
    _, mean, rstd = ops.layer_norm(one)
    want, _, _ = ops.layer_norm_backward(dy, one, None, mean, rstd)
    dx, _, _ = ops.layer_norm_backward(dy.expand(ROWS, cols), one.expand(ROWS, cols), None, mean.repeat(ROWS),
                                       rstd.repeat(ROWS))
    assert rows_are(dx, want)
    del dx
    torch.cuda.empty_cache()
