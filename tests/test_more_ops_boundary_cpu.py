"""Boundary of the operators that read documents in order (include/lda_ops.h: embedding, recurrence, distillation)
without a GPU: the argument structures and every refusal that comes before a device is touched."""
import ctypes
import os
import subprocess

import pytest

import paper_2007_08725_amd as lda

torch = pytest.importorskip("torch")
from paper_2007_08725_amd import ops  # noqa: E402
from test_ops_boundary_cpu import A, ARG, BACKWARD, BOTH, FORWARD, RANGE, ROOT, header, lib  # noqa: E402,F401

STRUCTS = (("lda_embed_args", ops.EmbedArgs), ("lda_recur_args", ops.RecurArgs), ("lda_distill_args", ops.DistillArgs))


def test_structures_follow_the_header(tmp_path):
    lines = []
    for struct, cls in STRUCTS:
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
    for struct, cls in STRUCTS:
        assert int(said[struct]) == ctypes.sizeof(cls)
        for field, _ in cls._fields_:
            assert int(said["%s.%s" % (struct, field)]) == getattr(cls, field).offset, field


def test_limits_follow_the_header():
    import re
    said = dict(re.findall(r"#define (LDA_OPS_\w+) (\d+)", header()))
    assert int(said["LDA_OPS_MAX_TOP"]) == ops.MAX_TOP and int(said["LDA_OPS_MAX_LISTED"]) == ops.MAX_LISTED
    assert int(said["LDA_OPS_RECUR_ROWS"]) == ops.RECUR_ROWS


def embed(**kw):
    return ops.EmbedArgs(**{**dict(dtype=1, rows=4, width=8, vocab=100, scale=1.0, words=A, weight=A, ld_weight=8, y=A,
                                   ldy=8, dy=A, lddy=8, dweight=A), **kw})


def recur(**kw):
    return ops.RecurArgs(**{**dict(dtype=1, rows=4, cols=8, docs=2, offsets=A, x=A, ldx=8, gate=A, ld_gate=8, h=A,
                                   ldh=8, last=A, kept=A, dh=A, lddh=8, dx=A, lddx=8, dgate=A, ld_dgate=8), **kw})


def distill(**kw):
    return ops.DistillArgs(**{**dict(dtype=1, rows=4, width=8, vocab=100, top=3, temperature=1.0, x=A, ldx=8, weight=A,
                                     ld_weight=8, words=A, ld_words=3, scores=A, ld_scores=3, loss=A, lse=A, logits=A,
                                     dloss=A, dx=A, lddx=8, dweight=A), **kw})


NAN, INF = float("nan"), float("inf")
CASES = [
    (embed, dict(dtype=3), ARG, BOTH), (embed, dict(dtype=-1), ARG, BOTH), (embed, dict(rows=-1), ARG, BOTH),
    (embed, dict(rows=ops.MAX_ROWS + 1), RANGE, BOTH), (embed, dict(width=0), ARG, BOTH),
    (embed, dict(width=ops.MAX_COLS + 1, ldy=1 << 21), RANGE, BOTH), (embed, dict(vocab=0), ARG, BOTH),
    (embed, dict(vocab=ops.MAX_VOCAB + 1), RANGE, BOTH), (embed, dict(scale=NAN), ARG, BOTH),
    (embed, dict(scale=INF), ARG, BOTH), (embed, dict(words=None), ARG, BOTH), (embed, dict(weight=None), ARG, FORWARD),
    (embed, dict(ld_weight=-1), ARG, FORWARD), (embed, dict(y=None), ARG, FORWARD), (embed, dict(ldy=7), ARG, FORWARD),
    (embed, dict(dy=None), ARG, BACKWARD), (embed, dict(lddy=-1), ARG, BACKWARD),
    (embed, dict(dweight=None), ARG, BACKWARD),
    (recur, dict(dtype=3), ARG, BOTH), (recur, dict(rows=-1), ARG, BOTH), (recur, dict(cols=0), ARG, BOTH),
    (recur, dict(rows=ops.MAX_ROWS + 1), RANGE, BOTH), (recur, dict(docs=-1), ARG, BOTH),
    (recur, dict(docs=ops.MAX_ROWS + 1), RANGE, BOTH), (recur, dict(offsets=None), ARG, BOTH),
    (recur, dict(rows=1 << 24, cols=1 << 20, ldh=1 << 20), RANGE, BOTH), (recur, dict(x=None), ARG, BOTH),
    (recur, dict(ldx=-1), ARG, BOTH), (recur, dict(gate=None), ARG, BOTH), (recur, dict(ld_gate=-1), ARG, BOTH),
    (recur, dict(kept=None), ARG, BOTH), (recur, dict(h=None), ARG, FORWARD), (recur, dict(ldh=7), ARG, FORWARD),
    (recur, dict(last=None), ARG, FORWARD), (recur, dict(dh=None), ARG, BACKWARD),
    (recur, dict(lddh=-1), ARG, BACKWARD), (recur, dict(dx=None), ARG, BACKWARD), (recur, dict(lddx=7), ARG, BACKWARD),
    (recur, dict(dgate=None), ARG, BACKWARD), (recur, dict(ld_dgate=7), ARG, BACKWARD),
    (recur, dict(state=A), ARG, BACKWARD), (recur, dict(dstate=A), ARG, BACKWARD),
    (distill, dict(dtype=3), ARG, BOTH), (distill, dict(rows=-1), ARG, BOTH), (distill, dict(width=0), ARG, BOTH),
    (distill, dict(vocab=0), ARG, BOTH), (distill, dict(vocab=ops.MAX_VOCAB + 1), RANGE, BOTH),
    (distill, dict(top=0), ARG, BOTH), (distill, dict(top=ops.MAX_TOP + 1), RANGE, BOTH),
    (distill, dict(rows=(1 << 20) + 1, top=256, ld_words=256, ld_scores=256), RANGE, BOTH),
    (distill, dict(rows=1 << 24, vocab=1 << 24), RANGE, BOTH), (distill, dict(temperature=0.0), ARG, BOTH),
    (distill, dict(temperature=-1.0), ARG, BOTH), (distill, dict(temperature=NAN), ARG, BOTH),
    (distill, dict(temperature=INF), ARG, BOTH), (distill, dict(temperature=1e-40), ARG, BOTH),
    (distill, dict(x=None), ARG, BOTH), (distill, dict(weight=None), ARG, BOTH), (distill, dict(words=None), ARG, BOTH),
    (distill, dict(ld_words=-1), ARG, BOTH), (distill, dict(scores=None), ARG, BOTH),
    (distill, dict(ld_scores=-1), ARG, BOTH), (distill, dict(lse=None), ARG, BOTH),
    (distill, dict(logits=None), ARG, BOTH), (distill, dict(loss=None), ARG, FORWARD),
    (distill, dict(dloss=None), ARG, BACKWARD), (distill, dict(dweight=None), ARG, BACKWARD),
    (distill, dict(dx=None), ARG, BACKWARD), (distill, dict(lddx=7), ARG, BACKWARD),
    (distill, dict(bias=A), ARG, BACKWARD), (distill, dict(dbias=A), ARG, BACKWARD),
]
NAMES = {embed: "lda_embedding", recur: "lda_recurrence", distill: "lda_softmax_distill"}


@pytest.mark.parametrize("case", range(len(CASES)))
def test_refusals(lib, case):  # noqa: F811
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


@pytest.mark.parametrize("change,status", [
    (dict(docs=2), ARG), (dict(rows=-1), ARG), (dict(state=None), ARG), (dict(last=None), ARG), (dict(x=None), ARG),
    (dict(gate=None), ARG), (dict(h=None), ARG), (dict(ldh=7), ARG), (dict(dtype=9), ARG), (dict(cols=0), ARG)])
def test_step_refusals(lib, change, status):  # noqa: F811
    a = recur(**{**dict(docs=4, state=A, offsets=None, kept=None), **change})
    assert ops._function("lda_recurrence_step")(ctypes.byref(a)) == status


@pytest.mark.parametrize("make", [embed, recur, distill])
@pytest.mark.parametrize("backward", [False, True])
def test_null_arguments(lib, make, backward):  # noqa: F811
    name = NAMES[make] + ("_backward" if backward else "")
    assert ops._function(name)(None) == ARG
    if name + "_workspace" in ops.EXPORTS:
        assert ops._function(name + "_workspace")(ctypes.byref(make()), None) == ARG
        assert ops._function(name + "_workspace")(None, ctypes.byref(ctypes.c_size_t())) == ARG
    assert ops._function("lda_recurrence_step")(None) == ARG


@pytest.mark.parametrize("make,change,backward", [
    (embed, dict(), True), (embed, dict(rows=20000), True), (recur, dict(), False), (recur, dict(), True),
    (distill, dict(), False), (distill, dict(rows=700), False), (distill, dict(), True),
    (distill, dict(bias=A, dbias=A), True)])
def test_workspace_is_checked(lib, make, change, backward):  # noqa: F811
    """A call whose workspace is missing, too small or misaligned is refused before any launch."""
    name = NAMES[make] + ("_backward" if backward else "")
    size = ctypes.c_size_t()
    a = make(**change)
    assert ops._function(name + "_workspace")(ctypes.byref(a), ctypes.byref(size)) == lda.LDA_OK and size.value > 0
    for workspace, bytes_ in ((None, size.value), (A, size.value - 1), (A + 8, size.value)):
        a = make(**change, workspace=workspace, workspace_bytes=bytes_)
        assert ops._function(name)(ctypes.byref(a)) == ARG


def test_workspace_grows_with_the_call(lib):  # noqa: F811
    """Every size in range has a workspace, the largest among them (counted in 64 bits)."""
    size = ctypes.c_size_t()
    for make, change in ((embed, dict(rows=ops.MAX_ROWS, width=1024, vocab=ops.MAX_VOCAB)),
                         (recur, dict(rows=ops.MAX_ROWS, cols=4096, ldx=4096, ld_gate=4096, lddh=4096, lddx=4096,
                                      ld_dgate=4096)),
                         (distill, dict(rows=1 << 20, top=256, vocab=100000))):
        a = make(**change)
        assert ops._function(NAMES[make] + "_backward_workspace")(ctypes.byref(a), ctypes.byref(size)) == lda.LDA_OK
        assert size.value > 1 << 27


def test_tensors_off_the_device_are_refused():
    x, words = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        ops.embedding(words, x)
    with pytest.raises(ValueError):
        ops.embedding_backward(x, words, 8)
    with pytest.raises(ValueError):
        ops.recurrence(x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        ops.recurrence_step(x, x, x)
    with pytest.raises(ValueError):
        ops.softmax_distill(x, x, words.view(2, 1), torch.zeros(2, 1))
