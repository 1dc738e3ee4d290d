"""What distillation's backward pass keeps of G (include/lda_ops.h), by the size of its workspace, without a GPU."""
import ctypes

import pytest

from test_more_ops_boundary_cpu import distill, lib, ops  # noqa: F401
import paper_2007_08725_amd as lda


def bytes_of(rows, vocab, width, dtype):
    size = ctypes.c_size_t()
    a = distill(dtype=dtype, rows=rows, width=width, vocab=vocab, ldx=width, ld_weight=width, lddx=width)
    assert ops._function("lda_softmax_distill_backward_workspace")(ctypes.byref(a), ctypes.byref(size)) == lda.LDA_OK
    return size.value


@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("width", [8, 1024])
def test_up_to_128_rows_keep_the_remainder(lib, dtype, width):  # noqa: F811
    """Two matrices of 16 bits, whatever tiles the vocabulary gives the products; beyond, one of at most 256 MiB."""
    for rows in (1, 16, 17, 63, 64, 65, 100, 127, 128):
        for vocab in (1, 8, 100, 1000, 8192, 30000, 141000, 1 << 20):
            words = min(-(-vocab // 64) * 64, (256 << 20) // (2 * rows) // 64 * 64)
            assert bytes_of(rows, vocab, width, dtype) >= 2 * 2 * rows * min(words, vocab), (rows, vocab)
    # the parts of dx differ by a row
    assert bytes_of(128, 1 << 20, width, dtype) - bytes_of(129, 1 << 20, width, dtype) > 128 << 20
