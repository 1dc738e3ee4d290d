"""Boundary of the word-model operators (include/lda_ops.h) without a GPU: the
exported symbols, the argument structures, and every refusal that comes before
a device is touched."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2007_08725_amd as lda

torch = pytest.importorskip("torch")
from paper_2007_08725_amd import ops  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lda.LIB_PATH):
        from paper_2007_08725_amd import _build
        _build.build()
    return lda.load_library()


def header():
    with open(os.path.join(ROOT, "include", "lda_ops.h")) as f:
        return re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)


def test_exports_every_declared_symbol(lib):
    declared = set(re.findall(r"\b(lda_[a-z_]+)\s*\(", header()))
    assert declared == set(ops.EXPORTS)
    for name in declared:
        assert hasattr(lib, name), name


def test_structures_follow_the_header(tmp_path):
    """Sizes and offsets of the binding's structures are the C compiler's."""
    lines = []
    for struct, cls in (("lda_norm_args", ops.NormArgs), ("lda_gated_args", ops.GatedArgs),
                        ("lda_xent_args", ops.XentArgs)):
        lines.append('printf("%%s %%zu\\n", "%s", sizeof(%s));' % (struct, struct))
        for field, _ in cls._fields_:
            lines.append('printf("%%s %%zu\\n", "%s.%s", offsetof(%s, %s));' % (struct, field, struct, field))
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include "lda_ops.h"\nint main(void) {\n%s\nreturn 0;\n}\n' % "\n".join(lines))
    exe = str(tmp_path / "offsets")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe],
                   check=True)
    said = dict(line.split() for line in subprocess.run([exe], capture_output=True, text=True, check=True)
                .stdout.splitlines())
    for struct, cls in (("lda_norm_args", ops.NormArgs), ("lda_gated_args", ops.GatedArgs),
                        ("lda_xent_args", ops.XentArgs)):
        assert int(said[struct]) == ctypes.sizeof(cls)
        for field, _ in cls._fields_:
            assert int(said["%s.%s" % (struct, field)]) == getattr(cls, field).offset, field


def test_limits_follow_the_header():
    said = dict(re.findall(r"#define (LDA_OPS_MAX_\w+) (\d+)", header()))
    assert int(said["LDA_OPS_MAX_ROWS"]) == ops.MAX_ROWS and int(said["LDA_OPS_MAX_COLS"]) == ops.MAX_COLS
    assert int(said["LDA_OPS_MAX_VOCAB"]) == ops.MAX_VOCAB and int(said["LDA_OPS_MAX_TILES"]) == ops.MAX_TILES


# pointers that are checked, never followed
A = 1 << 20


def norm(**kw):
    return ops.NormArgs(**{**dict(dtype=1, rows=4, cols=8, eps=1e-5, x=A, ldx=8, y=A, ldy=8, mean=A, rstd=A, dy=A,
                                  lddy=8, dx=A, lddx=8), **kw})


def gated(**kw):
    return ops.GatedArgs(**{**dict(dtype=1, act=0, rows=4, width=8, hidden=16, x=A, ldx=8, w_gate=A, ld_gate=8,
                                   w_value=A, ld_value=8, h=A, ldh=16, dh=A, lddh=16, dx=A, lddx=8, dw_gate=A,
                                   dw_value=A), **kw})


def xent(**kw):
    return ops.XentArgs(**{**dict(dtype=1, rows=4, width=8, vocab=100, x=A, ldx=8, weight=A, ld_weight=8, labels=A,
                                  loss=A, lse=A, dloss=A, dx=A, lddx=8, dweight=A), **kw})


ARG, RANGE = lda.LDA_E_ARG, lda.LDA_E_RANGE
FORWARD, BACKWARD, BOTH = (False,), (True,), (False, True)
CASES = [
    (norm, dict(dtype=3), ARG, BOTH), (norm, dict(dtype=-1), ARG, BOTH), (norm, dict(rows=-1), ARG, BOTH),
    (norm, dict(rows=ops.MAX_ROWS + 1), RANGE, BOTH), (norm, dict(cols=0), ARG, BOTH),
    (norm, dict(cols=ops.MAX_COLS + 1, ldx=1 << 21, ldy=1 << 21, lddx=1 << 21), RANGE, BOTH),
    (norm, dict(x=None), ARG, BOTH), (norm, dict(ldx=-8), ARG, BOTH), (norm, dict(y=None), ARG, FORWARD),
    (norm, dict(ldy=7), ARG, FORWARD), (norm, dict(mean=None), ARG, BOTH), (norm, dict(rstd=None), ARG, BOTH),
    (norm, dict(weight=A), ARG, FORWARD), (norm, dict(bias=A), ARG, FORWARD), (norm, dict(eps=-1.0), ARG, FORWARD),
    (norm, dict(eps=float("nan")), ARG, FORWARD), (norm, dict(eps=float("inf")), ARG, FORWARD),
    (norm, dict(dy=None), ARG, BACKWARD), (norm, dict(dx=None), ARG, BACKWARD), (norm, dict(lddx=7), ARG, BACKWARD),
    (norm, dict(dweight=A), ARG, BACKWARD), (norm, dict(dbias=A), ARG, BACKWARD),
    (gated, dict(dtype=9), ARG, BOTH), (gated, dict(act=3), ARG, BOTH), (gated, dict(act=-1), ARG, BOTH),
    (gated, dict(rows=-1), ARG, BOTH), (gated, dict(width=0), ARG, BOTH), (gated, dict(hidden=0), ARG, BOTH),
    (gated, dict(x=None), ARG, BOTH), (gated, dict(w_gate=None), ARG, BOTH), (gated, dict(w_value=None), ARG, BOTH),
    (gated, dict(ld_gate=-1), ARG, BOTH), (gated, dict(h=None), ARG, FORWARD), (gated, dict(ldh=15), ARG, FORWARD),
    (gated, dict(dh=None), ARG, BACKWARD), (gated, dict(dx=None), ARG, BACKWARD), (gated, dict(lddx=7), ARG, BACKWARD),
    (gated, dict(dw_gate=None), ARG, BACKWARD), (gated, dict(dw_value=None), ARG, BACKWARD),
    (gated, dict(rows=1 << 24, hidden=1 << 20, ldh=1 << 20), RANGE, BOTH),
    (xent, dict(dtype=3), ARG, BOTH), (xent, dict(rows=-1), ARG, BOTH), (xent, dict(vocab=0), ARG, BOTH),
    (xent, dict(vocab=ops.MAX_VOCAB + 1), RANGE, BOTH), (xent, dict(rows=1 << 24, vocab=1 << 24), RANGE, BOTH),
    (xent, dict(width=0), ARG, BOTH), (xent, dict(x=None), ARG, BOTH), (xent, dict(weight=None), ARG, BOTH),
    (xent, dict(labels=None), ARG, BOTH), (xent, dict(lse=None), ARG, BOTH), (xent, dict(loss=None), ARG, FORWARD),
    (xent, dict(dloss=None), ARG, BACKWARD), (xent, dict(dweight=None), ARG, BACKWARD),
    (xent, dict(dx=None), ARG, BACKWARD), (xent, dict(lddx=7), ARG, BACKWARD),
    (xent, dict(bias=A), ARG, BACKWARD), (xent, dict(dbias=A), ARG, BACKWARD),
]
NAMES = {norm: "lda_layer_norm", gated: "lda_gated", xent: "lda_softmax_xent"}


@pytest.mark.parametrize("case", range(len(CASES)))
def test_refusals(lib, case):
    make, change, status, ways = CASES[case]
    for backward in ways:
        name = NAMES[make] + ("_backward" if backward else "")
        a = make(**change)
        assert ops._function(name)(ctypes.byref(a)) == status, (name, change)
        assert lib.lda_last_error(None)
        if name + "_workspace" in ops.EXPORTS:
            size = ctypes.c_size_t(7)
            assert ops._function(name + "_workspace")(ctypes.byref(a), ctypes.byref(size)) == status
            assert size.value == 7


@pytest.mark.parametrize("make,backward", [(norm, False), (norm, True), (gated, False), (gated, True), (xent, False),
                                           (xent, True)])
def test_null_arguments(lib, make, backward):
    name = NAMES[make] + ("_backward" if backward else "")
    assert ops._function(name)(None) == ARG
    if name + "_workspace" in ops.EXPORTS:
        assert ops._function(name + "_workspace")(ctypes.byref(make()), None) == ARG
        assert ops._function(name + "_workspace")(None, ctypes.byref(ctypes.c_size_t())) == ARG


@pytest.mark.parametrize("make,change,backward", [
    (norm, dict(weight=A, bias=A, dweight=A, dbias=A), True), (gated, dict(), True), (xent, dict(), True),
    (gated, dict(rows=40, width=7, ldx=7, ld_gate=7, ld_value=7), False), (xent, dict(rows=700), False)])
def test_workspace_is_checked(lib, make, change, backward):
    """A call whose workspace is missing, too small or misaligned is refused before any launch."""
    name = NAMES[make] + ("_backward" if backward else "")
    size = ctypes.c_size_t()
    a = make(**change)
    assert ops._function(name + "_workspace")(ctypes.byref(a), ctypes.byref(size)) == lda.LDA_OK and size.value > 0
    for workspace, bytes_ in ((None, size.value), (A, size.value - 1), (A + 8, size.value)):
        a = make(**change, workspace=workspace, workspace_bytes=bytes_)
        assert ops._function(name)(ctypes.byref(a)) == ARG


def test_tensors_off_the_device_are_refused():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        ops.layer_norm(x)
    with pytest.raises(ValueError):
        ops.gated(x, x, x)
    with pytest.raises(ValueError):
        ops.softmax_xent(x, x, torch.zeros(2, dtype=torch.int32))
