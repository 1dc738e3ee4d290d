"""Sizes of an embedding's gradient that one launch has no room for (2^32 threads: 1,024 for each 64 KiB that are
cleared, 64 for each part that is summed), refused without a GPU; the largest below them have a workspace."""
import ctypes
import re

import pytest

from test_more_ops_boundary_cpu import embed, header, lib, ops  # noqa: F401
from test_ops_boundary_cpu import RANGE  # noqa: E402
import paper_2007_08725_amd as lda


def asked(**kw):
    size, a = ctypes.c_size_t(), embed(**kw)
    return ops._function("lda_embedding_backward_workspace")(ctypes.byref(a), ctypes.byref(size)), size.value


def test_limits_are_the_launches():
    said = dict(re.findall(r"#define (LDA_OPS_MAX_EMBED_\w+) (\d+)", header()))
    # a workgroup beside those that clear
    assert 1024 * (-(-int(said["LDA_OPS_MAX_EMBED_BYTES"]) // 65536) + 1) < 2 ** 32
    # four parts a workgroup
    assert 256 * -(-int(said["LDA_OPS_MAX_EMBED_PARTS"]) // 4) < 2 ** 32


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2), (2, 2)])
def test_cleared(lib, dtype, size):  # noqa: F811
    vocab, width = 1 << 24, 255 * 64 // size
    assert vocab * width * size == 255 << 30
    for rows in (0, 4, 10000):
        assert asked(dtype=dtype, rows=rows, vocab=vocab, width=width, lddy=width)[0] == lda.LDA_OK
        assert asked(dtype=dtype, rows=rows, vocab=vocab, width=width + 1, lddy=width + 1)[0] == RANGE
        assert lib.lda_last_error(None)
    a = embed(dtype=dtype, vocab=vocab, width=width + 1, ld_weight=width + 1, ldy=width + 1, rows=0)
    assert ops._function("lda_embedding")(ctypes.byref(a)) == lda.LDA_OK  # the forward pass clears nothing


@pytest.mark.parametrize("dtype,rows", [(0, 1 << 23), (1, 1 << 24), (2, 1 << 24)])
def test_summed(lib, dtype, rows):  # noqa: F811
    width = 1 << 20
    status, size = asked(dtype=dtype, rows=rows - 512, vocab=3, width=width, lddy=0)
    assert status == lda.LDA_OK and size > 1 << 37
    assert asked(dtype=dtype, rows=rows, vocab=3, width=width, lddy=0)[0] == RANGE
