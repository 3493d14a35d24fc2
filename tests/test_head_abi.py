"""The head's and the adapters' entry points without a GPU: struct layouts
against the header as C99, every refusal that needs no device, and the bytes of
their workspaces."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_17310_amd import adapters, esopt, head

HERE = os.path.dirname(os.path.abspath(__file__))
E, ALIGN = esopt.ES_ERR_INVALID_ARG, esopt.ES_ERR_ALIGN
P = 0x100000                                               # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    return esopt.load()


def test_header_layouts_match_the_binding(lib, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    exe = str(tmp_path / "head_consumer")
    libdir = os.path.dirname(esopt.LIB_PATH)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I",
                    os.path.join(os.path.dirname(HERE), "include"),
                    os.path.join(HERE, "harness", "head_consumer.c"), "-L", libdir,
                    "-l:" + os.path.basename(esopt.LIB_PATH), "-Wl,-rpath," + libdir, "-o", exe],
                   check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    got = {l.split()[0]: l.split()[1:] for l in out.splitlines()}
    for name, cls, pack in (("es_head_score_t", esopt.EsHeadScore, head._SCORE),
                            ("es_head_gradient_t", esopt.EsHeadGradient, head._GRADIENT),
                            ("es_adapt_t", esopt.EsAdapt, adapters._ADAPT)):
        want = [str(ctypes.sizeof(cls))]
        for f, _ in cls._fields_:
            want += [f, str(getattr(cls, f).offset)]
        assert got[name] == want
        assert pack.size == ctypes.sizeof(cls)
    assert got["values"] == [str(head.ES_HEAD_BAD_ID), str(adapters.ES_ADAPT_BAD_INDEX)]
    assert got["score_null"] == got["gradient_null"] == got["adapt_null"] == [str(E)]
    assert got["bytes_null"] == ["0"]


def _score(**kw):
    d = dict(x=P, weight=2 * P, x_stride=64, w_stride=64, ids=3 * P, teacher=None, loss=None,
             logp=4 * P, lse=5 * P, status=None, workspace=6 * P, workspace_bytes=1 << 40, rows=10,
             vocab=1000, hidden=64, entries=1, scale=1.0, reserved=0)
    d.update(kw)
    return esopt.EsHeadScore(**d)


def _gradient(**kw):
    d = dict(x=P, weight=2 * P, x_stride=64, w_stride=64, ids=3 * P, teacher=None, logp=4 * P,
             lse=5 * P, grad=6 * P, d_x=7 * P, d_weight=8 * P, dx_stride=64, dw_stride=64, status=None,
             workspace=9 * P, workspace_bytes=1 << 40, rows=10, vocab=1000, hidden=64, entries=1,
             scale=1.0, reserved=0)
    d.update(kw)
    return esopt.EsHeadGradient(**d)


def _adapt(**kw):
    d = dict(x=P, weight=2 * P, out=3 * P, x_stride=64, w_stride=64, out_stride=96, a=4 * P, b=5 * P,
             scales=None, index=6 * P, status=None, workspace=7 * P, workspace_bytes=1 << 40, rows=10,
             inner=64, outer=96, members=3, rank=16, reserved=0)
    d.update(kw)
    return esopt.EsAdapt(**d)


BOTH = [(dict(rows=65537), E, "rows"), (dict(vocab=0), E, "vocab"), (dict(vocab=(1 << 24) + 1), E, "vocab"),
        (dict(rows=65536, vocab=(1 << 20) + 1), E, "rows times vocab"),
        (dict(hidden=0), E, "hidden"), (dict(hidden=65537), E, "hidden"), (dict(entries=0), E, "entries"),
        (dict(entries=257, teacher=P), E, "entries"), (dict(entries=2), E, "teacher"),
        (dict(scale=float("nan")), E, "scale"), (dict(scale=float("-inf")), E, "scale"),
        (dict(reserved=1), E, "reserved"), (dict(x_stride=(1 << 22) + 1), E, "stride"),
        (dict(w_stride=1 << 40), E, "stride"), (dict(x=None), E, "null"), (dict(weight=None), E, "null"),
        (dict(ids=None), E, "null"), (dict(x=P + 1), ALIGN, "aligned"), (dict(weight=P + 1), ALIGN, "aligned"),
        (dict(ids=P + 4), ALIGN, "aligned")]


@pytest.mark.parametrize("change,code,word", BOTH + [
    (dict(logp=None), E, "needed"), (dict(lse=None), E, "needed"), (dict(loss=P), E, "loss"),
    (dict(teacher=P), E, "loss"), (dict(logp=P + 2), ALIGN, "aligned"),
    (dict(status=P + 1), ALIGN, "aligned"), (dict(workspace=P + 128), ALIGN, "aligned")])
def test_score_refuses(lib, change, code, word):
    args = _score(**change)
    assert lib.es_head_score(ctypes.byref(args), None) == code
    assert word in esopt.last_error()


@pytest.mark.parametrize("change,code,word", BOTH + [
    (dict(logp=None), E, "null"), (dict(lse=None), E, "null"), (dict(grad=None), E, "null"),
    (dict(dx_stride=63), E, "overlap"), (dict(dw_stride=32), E, "overlap"),
    (dict(dx_stride=1 << 30), E, "stride"), (dict(rows=0), E, "no rows"),
    (dict(d_x=P + 1), ALIGN, "aligned"), (dict(d_weight=P + 1), ALIGN, "aligned"),
    (dict(grad=P + 2), ALIGN, "aligned"), (dict(workspace=P + 16), ALIGN, "aligned")])
def test_gradient_refuses(lib, change, code, word):
    args = _gradient(**change)
    assert lib.es_head_gradient(ctypes.byref(args), None) == code
    assert word in esopt.last_error()


@pytest.mark.parametrize("change,code,word", [
    (dict(rows=(1 << 20) + 1), E, "rows"), (dict(inner=0), E, "inner"), (dict(inner=60), E, "inner"),
    (dict(inner=65544), E, "inner"), (dict(outer=0), E, "outer"), (dict(outer=(1 << 20) + 1), E, "outer"),
    (dict(rows=1 << 17, outer=1 << 20, out_stride=1 << 20), E, "rows times outer"),
    (dict(members=0), E, "members"), (dict(members=65537), E, "members"), (dict(rank=0), E, "rank"),
    (dict(rank=4), E, "rank"), (dict(rank=136), E, "rank"), (dict(reserved=1), E, "reserved"),
    (dict(x_stride=1 << 23), E, "stride"), (dict(out_stride=1 << 23), E, "stride"),
    (dict(x=None), E, "null"), (dict(weight=None), E, "null"), (dict(out=None), E, "null"),
    (dict(a=None), E, "null"), (dict(b=None), E, "null"), (dict(index=None), E, "null"),
    (dict(out=P), E, "out is x"), (dict(out_stride=95), E, "overlap"), (dict(x=P + 1), ALIGN, "aligned"),
    (dict(weight=P + 8), ALIGN, "aligned"), (dict(w_stride=68), ALIGN, "aligned"),
    (dict(a=P + 8), ALIGN, "aligned"), (dict(b=P + 2), ALIGN, "aligned"),
    (dict(index=P + 2), ALIGN, "aligned"), (dict(workspace=P + 64), ALIGN, "workspace")])
def test_adapt_refuses(lib, change, code, word):
    args = _adapt(**change)
    assert lib.es_adapt_project(ctypes.byref(args), None) == code
    assert word in esopt.last_error()


def test_calls_without_rows_do_nothing(lib):
    assert lib.es_head_score(ctypes.byref(_score(rows=0)), None) == 0
    assert lib.es_head_gradient(ctypes.byref(_gradient(rows=0, d_weight=None)), None) == 0
    assert lib.es_adapt_project(ctypes.byref(_adapt(rows=0)), None) == 0


def test_workspaces_do_not_hold_the_logits(lib):
    """A few numbers a row and tile of 256 tokens for scores; for gradients a
    bounded piece of the logits', whatever the vocabulary."""
    for fn, make in ((lib.es_head_score_bytes, _score), (lib.es_head_gradient_bytes, _gradient)):
        assert fn(ctypes.byref(make(rows=0))) == 0
        assert fn(ctypes.byref(make(hidden=0))) == 0
        assert 0 < fn(ctypes.byref(make()))
    rows, vocab, hidden = 4096, 151936, 5120
    size = dict(rows=rows, vocab=vocab, hidden=hidden, x_stride=hidden, w_stride=hidden)
    packed = 2 * rows * hidden
    score = lib.es_head_score_bytes(ctypes.byref(_score(**size)))
    assert score <= packed + 8 * rows * (vocab // 256 + 1) + (1 << 20)
    grad = lib.es_head_gradient_bytes(ctypes.byref(_gradient(dx_stride=hidden, dw_stride=hidden, **size)))
    assert grad <= packed + (1 << 28) + 4 * 4 * rows * hidden + (1 << 20)
    # rows that are not word-aligned: a bounded copy of a piece of the head
    size.update(hidden=5119)
    more = lib.es_head_score_bytes(ctypes.byref(_score(**size)))
    assert score < more <= score + (1 << 28) + (1 << 20)


def test_workspaces_that_are_too_small_are_refused(lib):
    """Before the device is asked for anything but its number."""
    for fn, make in ((lib.es_head_score, _score), (lib.es_head_gradient, _gradient),
                     (lib.es_adapt_project, _adapt)):
        rc = fn(ctypes.byref(make(workspace_bytes=255)), None)
        assert rc in (E, esopt.ES_ERR_HIP) and (rc != E or "workspace" in esopt.last_error())


def test_the_stride_of_a_single_row_is_not_looked_at(lib):
    """A row taken out of a larger array, or a column seen as a row, has any stride: the
    workspace is that of rows side by side, and the call gets as far as the device."""
    any_ = (0, 1, 3, 68, (1 << 22) + 8, 1 << 60)
    for fn, size, make, one in (
            (lib.es_head_score, lib.es_head_score_bytes, _score, [("rows", "x_stride"), ("vocab", "w_stride")]),
            (lib.es_head_gradient, lib.es_head_gradient_bytes, _gradient,
             [("rows", "x_stride"), ("rows", "dx_stride"), ("vocab", "w_stride"), ("vocab", "dw_stride")]),
            (lib.es_adapt_project, lib.es_adapt_bytes, _adapt,
             [("rows", "x_stride"), ("rows", "out_stride"), ("outer", "w_stride")])):
        for rows, stride in one:
            want = size(ctypes.byref(make(**{rows: 1})))
            assert want > 0
            for n in any_:
                args = make(**{rows: 1, stride: n})
                assert size(ctypes.byref(args)) == want, (rows, stride, n)
                # with too little workspace the call ends on the host, with a GPU and without
                args.workspace_bytes = 1
                assert fn(ctypes.byref(args), None) in (E, esopt.ES_ERR_HIP)
                said = esopt.last_error()
                assert "stride" not in said and "overlap" not in said and "aligned" not in said


@pytest.mark.parametrize("change,refused", [
    (dict(out=P + 16), True), (dict(out=P - 2 * 96 * 9), True),              # over x's rows
    (dict(out=P + 2 * 64 * 10, out_stride=96), False), (dict(out=P - 2 * 96 * 10), False),   # beside them
    # within common rows of 160: columns 64 .. 159 beside 0 .. 63, and one too early or too late
    (dict(x_stride=160, out_stride=160, out=P + 2 * 64), False),
    (dict(x_stride=160, out_stride=160, out=P + 2 * 63), True),
    (dict(x_stride=160, out_stride=160, out=P + 2 * 65), True),
    (dict(x_stride=160, out_stride=160, out=P - 2 * 96), False),
    (dict(x_stride=160, out_stride=160, out=P - 2 * 95), True),
    (dict(x_stride=160, out_stride=160, out=P + 2 * 160 * 9 + 2 * 64), False),
    (dict(x_stride=160, out_stride=160, out=P + 2 * 160 * 4 + 2 * 60), True),
    (dict(rows=1, out=P + 2 * 64), False), (dict(rows=1, out=P + 2 * 63), True),
    (dict(rows=1, out=P - 2 * 96), False), (dict(rows=1, out=P - 2 * 95), True),
    (dict(out=2 * P), True), (dict(out=2 * P + 2 * 95 * 64), True), (dict(out=2 * P + 2 * 96 * 64), False),
    (dict(out=4 * P), True), (dict(out=4 * P + 2 * 3 * 16 * 64), False),
    (dict(out=5 * P + 2 * 3 * 16 * 96 - 2), True), (dict(out=5 * P + 2 * 3 * 16 * 96), False)])
def test_an_output_over_an_input_is_refused(lib, change, refused):
    """Whose rows would be read after they are written."""
    args = _adapt(**change)
    assert (lib.es_adapt_bytes(ctypes.byref(args)) == 0) == refused
    args.workspace_bytes = 1
    rc = lib.es_adapt_project(ctypes.byref(args), None)
    assert (rc == E and "shares memory" in esopt.last_error()) == refused
