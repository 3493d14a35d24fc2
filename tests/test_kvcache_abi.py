"""The cache's entry points without a GPU: struct layouts against the header
as C99, and every refusal that needs no device."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2608_17310_amd import esopt
from paper_2608_17310_amd import kvcache as kvc

HERE = os.path.dirname(os.path.abspath(__file__))
E = esopt.ES_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    return esopt.load()


def test_header_layouts_match_the_binding(lib, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    exe = str(tmp_path / "kv_consumer")
    libdir = os.path.dirname(esopt.LIB_PATH)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I",
                    os.path.join(os.path.dirname(HERE), "include"),
                    os.path.join(HERE, "harness", "kv_consumer.c"), "-L", libdir,
                    "-l:" + os.path.basename(esopt.LIB_PATH), "-Wl,-rpath," + libdir, "-o", exe],
                   check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    got = {l.split()[0]: l.split()[1:] for l in out.splitlines()}
    for name, cls in (("es_kv_desc_t", esopt.EsKvDesc), ("es_kv_append_t", esopt.EsKvAppend),
                      ("es_kv_attend_t", esopt.EsKvAttend)):
        want = [str(ctypes.sizeof(cls))]
        for f, _ in cls._fields_:
            want += [f, str(getattr(cls, f).offset)]
        assert got[name] == want
    assert got["values"] == [str(v) for v in (
        kvc.ES_KV_INT8, kvc.ES_KV_E4M3, kvc.ES_KV_BF16, kvc.ES_KV_ADJACENT, kvc.ES_KV_BAD_SLOT,
        kvc.ES_KV_BAD_POSITION, kvc.ES_KV_BAD_PAGE, kvc.ES_KV_BAD_LENGTH)]
    assert kvc._APPEND.size == ctypes.sizeof(esopt.EsKvAppend)
    assert kvc._ATTEND.size == ctypes.sizeof(esopt.EsKvAttend)
    assert got["create_null"] == [str(E)] and got["attend_null"] == [str(E)]
    assert got["destroy_null"] == ["0"]


def _desc(**kw):
    d = dict(k_pages=0x100000, v_pages=0x200000, k_scales=0x300000, v_scales=0x400000, n_pages=4,
             page=64, kv_heads=2, head_dim=64, format=kvc.ES_KV_INT8, reserved=0)
    d.update(kw)
    return esopt.EsKvDesc(**d)


@pytest.mark.parametrize("change,code,word", [
    (dict(format=3), E, "format"), (dict(reserved=1), E, "reserved"),
    (dict(page=32), E, "page"), (dict(page=96), E, "page"), (dict(page=2048), E, "page"),
    (dict(n_pages=0), E, "n_pages"), (dict(n_pages=(1 << 25) + 1), E, "n_pages"),
    (dict(kv_heads=0), E, "kv_heads"), (dict(kv_heads=1025), E, "kv_heads"),
    (dict(head_dim=96), E, "head_dim"), (dict(head_dim=512), E, "head_dim"),
    (dict(k_pages=None), E, "null"), (dict(v_pages=None), E, "null"),
    (dict(v_scales=None), E, "null"), (dict(format=kvc.ES_KV_BF16), E, "no scales"),
    (dict(k_pages=0x100008), esopt.ES_ERR_ALIGN, "aligned"),
    (dict(v_scales=0x400004), esopt.ES_ERR_ALIGN, "aligned")])
def test_create_refuses(lib, change, code, word):
    h = ctypes.c_void_p()
    d = _desc(**change)
    assert lib.es_kv_create(ctypes.byref(d), ctypes.byref(h)) == code
    assert word in esopt.last_error() and not h.value
    assert lib.es_kv_create(ctypes.byref(d), None) == E


class FakeCache(ctypes.Structure):
    """The head of the library's handle: device, then the description."""
    _fields_ = [("device", ctypes.c_int), ("d", esopt.EsKvDesc)]


@pytest.fixture
def fake():
    return FakeCache(0, _desc())


def _append(**kw):
    a = dict(q=0x10000, k=0x20000, v=0x30000, q_out=0x40000, q_stride=256, k_stride=128, v_stride=128,
             q_out_stride=256, q_gain=0x50000, k_gain=0x50000, rope=0x60000, positions=0x70000,
             slots=0x80000, status=None, tokens=3, q_heads=4, rot=64, rope_rows=10, eps=1e-6, flags=0)
    a.update(kw)
    return esopt.EsKvAppend(**a)


@pytest.mark.parametrize("change,code,word", [
    (dict(tokens=(1 << 24) + 1), E, "tokens"), (dict(q_heads=1025), E, "q_heads"),
    (dict(flags=2), E, "flags"), (dict(rot=8), E, "rot"), (dict(rot=80), E, "rot"),
    (dict(eps=0.0), E, "eps"), (dict(eps=float("nan")), E, "eps"), (dict(eps=float("inf")), E, "eps"),
    (dict(rope=None), E, "rotation"), (dict(positions=None), E, "rotation"),
    (dict(rope_rows=0), E, "rotation"), (dict(k=None), E, "null"), (dict(v=None), E, "null"),
    (dict(slots=None), E, "null"), (dict(q=None), E, "null"), (dict(q_out=None), E, "null"),
    (dict(q_out_stride=255), E, "overlap"), (dict(k=0x20001), esopt.ES_ERR_ALIGN, "aligned"),
    (dict(slots=0x80004), esopt.ES_ERR_ALIGN, "aligned"), (dict(rope=0x60002), esopt.ES_ERR_ALIGN, "aligned"),
    (dict(status=0x90002), esopt.ES_ERR_ALIGN, "aligned")])
def test_append_refuses(lib, fake, change, code, word):
    a = _append(**change)
    assert lib.es_kv_append(ctypes.byref(fake), ctypes.byref(a), None) == code
    assert word in esopt.last_error()


def test_append_of_nothing_is_a_no_op(lib, fake):
    a = _append(tokens=0, k=None, v=None, q=None)
    assert lib.es_kv_append(ctypes.byref(fake), ctypes.byref(a), None) == esopt.ES_OK
    assert lib.es_kv_append(None, ctypes.byref(a), None) == E
    assert lib.es_kv_append(ctypes.byref(fake), None, None) == E


def test_read_refuses(lib, fake):
    R = lib.es_kv_read
    h = ctypes.byref(fake)
    assert R(None, 0x1000, 1, 0x2000, 128, 0x3000, 128, None, None) == E
    assert R(h, 0x1000, (1 << 24) + 1, 0x2000, 128, 0x3000, 128, None, None) == E
    assert R(h, None, 2, 0x2000, 128, 0x3000, 128, None, None) == E
    assert R(h, 0x1000, 2, None, 128, 0x3000, 128, None, None) == E
    assert R(h, 0x1000, 2, 0x2000, 127, 0x3000, 128, None, None) == E
    assert R(h, 0x1000, 2, 0x2000, 128, 0x3001, 128, None, None) == esopt.ES_ERR_ALIGN
    assert R(h, None, 0, None, 0, None, 0, None, None) == esopt.ES_OK


def _attend(**kw):
    a = dict(q=0x10000, out=0x20000, q_stride=256, out_stride=256, tables=0x30000, lengths=0x40000,
             starts=0x50000, first=None, limit=None, slopes=None, status=None, rows=3, n_seqs=2,
             table_stride=5, q_heads=4, max_rows=2, max_length=100, scale=0.125, cap=0.0)
    a.update(kw)
    return esopt.EsKvAttend(**a)


@pytest.mark.parametrize("change,code,word", [
    (dict(rows=(1 << 24) + 1), E, "rows"), (dict(n_seqs=0), E, "n_seqs"),
    (dict(n_seqs=65537), E, "n_seqs"), (dict(q_heads=0), E, "q_heads"), (dict(q_heads=3), E, "q_heads"),
    (dict(q_heads=130), E, "q_heads"), (dict(scale=float("inf")), E, "scale"),
    (dict(scale=float("nan")), E, "scale"), (dict(cap=-1.0), E, "cap"),
    (dict(cap=float("nan")), E, "cap"), (dict(cap=1e-20), E, "cap"), (dict(cap=float("inf")), E, "cap"),
    (dict(table_stride=0), E, "table_stride"), (dict(q=None), E, "null"), (dict(out=None), E, "null"),
    (dict(tables=None), E, "null"), (dict(lengths=None), E, "null"), (dict(starts=None), E, "null"),
    (dict(out_stride=255), E, "overlap"), (dict(out=0x20001), esopt.ES_ERR_ALIGN, "aligned"),
    (dict(first=0x60002), esopt.ES_ERR_ALIGN, "aligned"),
    (dict(slopes=0x60001), esopt.ES_ERR_ALIGN, "aligned")])
def test_attend_refuses(lib, fake, change, code, word):
    a = _attend(**change)
    assert lib.es_kv_attend(ctypes.byref(fake), ctypes.byref(a), None) == code
    assert word in esopt.last_error()


def test_attend_of_no_rows_is_a_no_op(lib, fake):
    a = _attend(rows=0, q=None, out=None)
    assert lib.es_kv_attend(ctypes.byref(fake), ctypes.byref(a), None) == esopt.ES_OK
    assert lib.es_kv_device_bytes(None) == 0


def test_binding_refuses_shapes_and_types():
    bf = torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        kvc.KVCache(bf, bf)
    with pytest.raises(ValueError, match="bfloat16"):
        kvc.KVCache(bf.float(), bf.float())
    with pytest.raises(ValueError, match="shape"):
        kvc.KVCache(bf, bf[:, :1])
    with pytest.raises(ValueError, match="format"):
        kvc.KVCache.allocate(1, 1, 64, "fp4", device="cpu")


def test_strides_whose_extent_leaves_64_bits_are_refused(lib, fake):
    """2^23 rows of 2^40 elements are 2^64 bytes: an extent that wraps to a few
    bytes would pass the check of the allocation.  No device is asked."""
    h, n, far = ctypes.byref(fake), (1 << 23) + 1, 1 << 40
    for name in ("q_stride", "k_stride", "v_stride", "q_out_stride"):
        for stride in (far, (1 << 38) + 1, (1 << 64) - 1):
            a = _append(tokens=n, **{name: stride})
            assert lib.es_kv_append(h, ctypes.byref(a), None) == E, name
            assert "stride" in esopt.last_error()
    for strides in ((far, 128), (128, far)):
        assert lib.es_kv_read(h, 0x1000, n, 0x2000, strides[0], 0x3000, strides[1], None, None) == E
        assert "stride" in esopt.last_error()
    for name in ("q_stride", "out_stride"):
        a = _attend(rows=n, **{name: far})
        assert lib.es_kv_attend(h, ctypes.byref(a), None) == E
        assert "stride" in esopt.last_error()


def test_calls_beyond_a_launch_are_refused(lib, fake):
    """A launch has fewer than 2^32 lanes: more tokens than it can take are
    refused before any device is asked."""
    n = 1 << 24
    a = _append(tokens=n, q_heads=1024, q_stride=1024 * 64, q_out_stride=1024 * 64)
    assert lib.es_kv_append(ctypes.byref(fake), ctypes.byref(a), None) == E
    assert "too many tokens" in esopt.last_error()
    wide = FakeCache(0, _desc(kv_heads=1024))
    a = _append(tokens=n, q=None, q_out=None, q_heads=0)
    assert lib.es_kv_append(ctypes.byref(wide), ctypes.byref(a), None) == E
    assert "too many tokens" in esopt.last_error()
    row = 1024 * 64
    assert lib.es_kv_read(ctypes.byref(wide), 0x1000, n, 0x2000, row, 0x3000, row, None, None) == E
    assert "too many tokens" in esopt.last_error()
