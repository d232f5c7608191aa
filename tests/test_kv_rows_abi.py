"""Refusals and host bookkeeping of the paged cache's operators (laser_kv_append / truncate / write / read,
laser_attend) through the C ABI, without a device: handles over pointers that are never followed, and a
model that is not finalized, so that a call whose arguments are in order ends with STATE."""
import ctypes as C
import math

import pytest

from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd.configs import ModelShape

PTR = 1 << 20


def _kv(kind="int8", pool=PTR, pages=64, seqs=4, per_seq=32, layers=2):
    shape = ModelShape("abi", layers, 64, 4, 2, 64, 64, 64, True, False, "f32" if kind == "f32" else "bf16", 1.0e4, 1.0e-5,
                       kind if kind in ("fp8", "int8") else "")
    desc = L.desc_from_shape(shape, 1024)
    m, kv = C.c_void_p(), C.c_void_p()
    L._call("laser_model_create", C.byref(desc), C.byref(m))
    L._call("laser_kv_create", m, pages, seqs, per_seq, pool, pool + (1 << 24), pool + (1 << 25), C.byref(kv))
    return m, kv


def _code(name, *args):
    return getattr(L.lib(), name)(*args)


def _msg():
    return L.lib().laser_last_error().decode()


def _rows(n, heads, dtype=L.DTYPE_BF16, ptr=PTR, row=None, head=64):
    return L.laser_rows(ptr, dtype, n, heads * 64 if row is None else row, head)


def test_int8_pool_bytes():
    m, _ = _kv()
    nb = C.c_size_t()
    L._call("laser_kv_pool_bytes", m, 10, C.byref(nb))
    assert nb.value == 2 * 10 * 2 * (16 * 64 + 16 * 4)


def test_int8_needs_bf16_weights():
    shape = ModelShape("abi", 1, 64, 4, 2, 64, 64, 64, True, False, "f32", 1.0e4, 1.0e-5, "int8")
    desc, m = L.desc_from_shape(shape, 1024), C.c_void_p()
    assert _code("laser_model_create", C.byref(desc), C.byref(m)) == L.ERR_UNSUPPORTED
    desc.kv_dtype = 4
    assert _code("laser_model_create", C.byref(desc), C.byref(m)) == L.ERR_INVALID_ARG


def test_int8_pools_are_aligned():
    with pytest.raises(L.LaserError, match="16-byte aligned") as e:
        _kv(pool=PTR + 8)
    assert e.value.code == L.ERR_UNSUPPORTED


def test_append_and_truncate():
    _, kv = _kv(pages=6)
    L._call("laser_kv_add_seq", kv, 0, 15)
    L._call("laser_kv_append", kv, 0, 2)
    buf, n = (C.c_int32 * 32)(), C.c_int()

    def table():
        L._call("laser_kv_page_table", kv, 0, buf, 32, C.byref(n))
        return list(buf[:n.value])

    assert table() == [0, 1]
    assert _code("laser_kv_append", kv, 0, 5 * 16) == L.ERR_OUT_OF_PAGES and table() == [0, 1]
    assert _code("laser_kv_append", kv, 0, -1) == L.ERR_INVALID_ARG
    assert _code("laser_kv_append", kv, 1, 1) == L.ERR_INVALID_ARG
    assert _code("laser_kv_append", kv, 0, 2 ** 31 - 1) == L.ERR_INVALID_ARG
    assert _code("laser_kv_truncate", kv, 0, 18) == L.ERR_INVALID_ARG
    L._call("laser_kv_truncate", kv, 0, 16)
    assert table() == [0]
    L._call("laser_kv_append", kv, 0, 1)
    assert table() == [0, 1]
    assert _code("laser_kv_truncate", None, 0, 1) == L.ERR_STATE


def test_append_after_the_model_is_gone():
    m, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 15)
    L._call("laser_model_destroy", m)
    assert _code("laser_kv_append", kv, 0, 1) == L.ERR_STATE
    L._call("laser_kv_truncate", kv, 0, 3)  # (host bookkeeping alone)


def _write(kv, runs, k, v, layer=0, fn="laser_kv_write"):
    arr = (L.laser_kv_run * max(1, len(runs)))(*runs)
    return _code(fn, kv, layer, len(runs), arr, C.byref(k), C.byref(v), None)


@pytest.mark.parametrize("fn", ["laser_kv_write", "laser_kv_read"])
def test_rows_refusals(fn):
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 40)
    L._call("laser_kv_add_seq", kv, 1, 20)
    good, also = _rows(64, 2), _rows(64, 2, ptr=2 * PTR)
    ok = [L.kv_run(0, 3, 20, 5)]
    assert _write(kv, ok, good, also, fn=fn) == L.ERR_STATE and "finalized" in _msg()  # the arguments are in order

    def refused(code, runs=ok, k=good, v=also, layer=0):
        assert _write(kv, runs, k, v, layer, fn) == code, _msg()

    for layer in (-1, 2):
        refused(L.ERR_INVALID_ARG, layer=layer)
    refused(L.ERR_INVALID_ARG, [L.kv_run(2, 0, 1)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(-1, 0, 1)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 30, 11)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, -1, 2)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 0, -1)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 0, 10, 55)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 0, 10, -1)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 2 ** 31 - 1, 1)])
    refused(L.ERR_INVALID_ARG, [L.kv_run(0, 0, 1, 2 ** 31 - 1)])
    refused(L.ERR_INVALID_ARG, k=_rows(64, 2, ptr=0))
    refused(L.ERR_INVALID_ARG, k=_rows(64, 2, ptr=PTR + 1))
    refused(L.ERR_INVALID_ARG, v=_rows(64, 2, row=-128))
    refused(L.ERR_INVALID_ARG, v=_rows(-1, 2))
    refused(L.ERR_UNSUPPORTED, v=_rows(64, 2, dtype=L.DTYPE_FP8_E4M3))
    refused(L.ERR_UNSUPPORTED, v=_rows(64, 2, dtype=L.DTYPE_F32))
    twice = [L.kv_run(0, 3, 20, 0), L.kv_run(0, 22, 2, 30)]     # position 22 twice
    same_row = [L.kv_run(0, 3, 10, 0), L.kv_run(1, 0, 5, 9)]    # row 9 twice
    flat = _rows(64, 2, row=64, head=64)                        # heads of a row overlap the next row
    if fn == "laser_kv_write":
        refused(L.ERR_INVALID_ARG, twice)
        refused(L.ERR_STATE, same_row)  # (the same row written to two places is fine)
        refused(L.ERR_STATE, k=flat)
        refused(L.ERR_STATE, k=_rows(64, 2, row=0, head=0))
    else:
        refused(L.ERR_INVALID_ARG, v=good)  # both into the same place
        refused(L.ERR_STATE, twice)
        refused(L.ERR_INVALID_ARG, same_row)
        refused(L.ERR_INVALID_ARG, k=flat)
        refused(L.ERR_INVALID_ARG, k=_rows(64, 2, row=0))
        refused(L.ERR_STATE, k=_rows(64, 2, row=64, head=64 * 64))
    assert _write(None, ok, good, good, fn=fn) == L.ERR_STATE
    _, odd = _kv("bf16", pool=PTR + 8)
    L._call("laser_kv_add_seq", odd, 0, 40)
    assert _write(odd, ok, good, good, fn=fn) == L.ERR_UNSUPPORTED


def test_overlap_of_far_rows():
    """rows - 1 times a row stride of 2^40 passes 64 bits: not taken for rows that lie within heads."""
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 40)
    run = [L.kv_run(0, 0, 1)]
    also = _rows(4, 2, ptr=2 * PTR)
    # two heads 2^39 apart, rows 2^40 apart: apart; rows 2^38 apart: row 2 of head 0 is row 0 of head 1
    assert _write(kv, run, _rows(2 ** 30, 2, row=2 ** 40, head=2 ** 39), also, fn="laser_kv_read") == L.ERR_STATE
    assert _write(kv, run, _rows(2 ** 25 + 1, 2, row=2 ** 39, head=2 ** 40), also, fn="laser_kv_read") == L.ERR_INVALID_ARG
    assert _write(kv, run, _rows(3, 2, row=2 ** 38, head=2 ** 39), also, fn="laser_kv_read") == L.ERR_INVALID_ARG
    assert _write(kv, run, _rows(2, 2, row=2 ** 38, head=2 ** 39), also, fn="laser_kv_read") == L.ERR_STATE


def test_write_into_a_shared_page_is_refused():
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 32)
    assert _code("laser_kv_fork", kv, 0, 1, None) == L.ERR_STATE  # (a fork wants a finalized model)


def _attend(kv, spans, q, o, layer=0, scale=0.125, causal=1, window=0, lse=None, ws=None, nb=0):
    arr = (L.laser_attend_span * max(1, len(spans)))(*spans)
    return _code("laser_attend", kv, layer, len(spans), arr, scale, causal, window, C.byref(q), C.byref(o), lse, ws, nb, None)


def _bytes(kv, spans, dtype=L.DTYPE_BF16, causal=1, window=0):
    arr = (L.laser_attend_span * max(1, len(spans)))(*spans)
    nb = C.c_size_t(12345)
    code = _code("laser_attend_workspace", kv, len(spans), arr, dtype, causal, window, C.byref(nb))
    return code, nb.value


def test_attend_refusals():
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 400)
    L._call("laser_kv_add_seq", kv, 1, 0)
    good = _rows(64, 4)
    ok = [L.attend_span(0, 10, 90, row0=3, kv_end=100), L.attend_span(1, 1, 0, row0=20)]
    assert _attend(kv, ok, good, good) == L.ERR_STATE and "finalized" in _msg()

    def refused(code, spans=ok, q=good, o=good, **kw):
        assert _attend(kv, spans, q, o, **kw) == code, _msg()

    for layer in (-1, 2):
        refused(L.ERR_INVALID_ARG, layer=layer)
    for scale in (math.nan, math.inf):
        refused(L.ERR_INVALID_ARG, scale=scale)
    refused(L.ERR_INVALID_ARG, window=-1)
    refused(L.ERR_INVALID_ARG, lse=PTR + 2)
    S = L.attend_span
    for bad in (S(2, 1, 0), S(0, -1, 0), S(0, 1, -1), S(0, 1, 0, row0=-1), S(0, 1, 0, kv_begin=-1), S(0, 1, 0, kv_end=401),
                S(0, 1, 0, kv_end=-2), S(0, 1, 0, kv_begin=5, kv_end=4), S(0, 10, 0, row0=55), S(0, 65, 0),
                S(0, 1, 2 ** 31 - 1), S(0, 1, 0, row0=2 ** 31 - 1), S(0, 2 ** 31 - 1, 0), S(0, 2 ** 26 + 1, 0)):
        refused(L.ERR_INVALID_ARG, [bad])
    refused(L.ERR_INVALID_ARG, [S(0, 10, 0), S(0, 3, 0, row0=9)])
    refused(L.ERR_INVALID_ARG, q=_rows(64, 4, ptr=0))
    refused(L.ERR_INVALID_ARG, q=_rows(20, 4))
    refused(L.ERR_INVALID_ARG, o=_rows(64, 4, row=128))
    refused(L.ERR_UNSUPPORTED, o=_rows(64, 4, dtype=L.DTYPE_F32))
    refused(L.ERR_UNSUPPORTED, q=_rows(64, 4, dtype=L.DTYPE_INT8), o=_rows(64, 4, dtype=L.DTYPE_INT8))
    refused(L.ERR_STATE, q=_rows(64, 4, row=0, head=0), o=_rows(64, 4, ptr=2 * PTR))  # (queries may be broadcast)
    assert _attend(None, ok, good, good) == L.ERR_STATE


def test_attend_in_place_wants_the_same_strides():
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 40)
    span = [L.attend_span(0, 4, 10)]
    q = _rows(64, 4)
    assert _attend(kv, span, q, _rows(64, 4)) == L.ERR_STATE and "finalized" in _msg()
    assert _attend(kv, span, q, _rows(64, 4, row=512)) == L.ERR_INVALID_ARG
    assert _attend(kv, span, q, _rows(64, 4, row=64, head=64 * 64)) == L.ERR_INVALID_ARG
    assert _attend(kv, span, q, _rows(64, 4, row=512, ptr=2 * PTR)) == L.ERR_STATE


def test_attend_workspace():
    """Short keys need none; long ones (rows + 2) floats per row, head and split; a call without it is refused."""
    _, kv = _kv(pages=64, per_seq=64)
    L._call("laser_kv_add_seq", kv, 0, 1000)
    L._call("laser_kv_add_seq", kv, 1, 16)
    S = L.attend_span
    assert _bytes(kv, []) == (L.OK, 0)
    assert _bytes(kv, [S(1, 1, 15)]) == (L.OK, 0)
    assert _bytes(kv, [S(0, 1, 999, kv_begin=990)]) == (L.OK, 0)
    assert _bytes(kv, [S(0, 1, 999)], window=100) == (L.OK, 0)
    assert _bytes(kv, [S(0, 1, 20)]) == (L.OK, 0) and _bytes(kv, [S(0, 1, 20)], causal=0)[1] > 0
    code, nb = _bytes(kv, [S(0, 1, 999)])
    assert code == L.OK and nb > 0 and nb <= 4 * 128 * (64 + 2) * 4 + 256
    q = _rows(64, 4)
    assert _attend(kv, [S(0, 1, 999)], q, q) == L.ERR_INVALID_ARG and str(nb) in _msg()
    assert _attend(kv, [S(0, 1, 999)], q, q, ws=PTR, nb=nb - 1) == L.ERR_INVALID_ARG
    assert _attend(kv, [S(0, 1, 999)], q, q, ws=PTR + 4, nb=nb) == L.ERR_INVALID_ARG
    assert _attend(kv, [S(0, 1, 999)], q, q, ws=PTR, nb=nb) == L.ERR_STATE
    assert _bytes(kv, [S(0, 1, 999)], dtype=L.DTYPE_FP8_E4M3)[0] == L.ERR_UNSUPPORTED
    assert _bytes(kv, [S(3, 1, 0)])[0] == L.ERR_INVALID_ARG


def test_attend_rows_beyond_a_grid():
    """A launch has fewer than 2^32 threads: 2^26 rows of 2 heads per kv head are 2^23 tiles of 16 columns, 2 kv heads,
    256 threads.  Refused before anything is launched."""
    _, kv = _kv("f32")
    L._call("laser_kv_add_seq", kv, 0, 40)
    most = [L.attend_span(0, 2 ** 26 - 16, 0, kv_end=8)]
    assert _bytes(kv, most, L.DTYPE_F32)[0] == L.OK
    q, ws = _rows(2 ** 26, 4, dtype=L.DTYPE_F32), _bytes(kv, most, L.DTYPE_F32)[1]
    assert ws == 0 and _attend(kv, most, q, q) == L.ERR_STATE and "finalized" in _msg()
    over = [L.attend_span(0, 2 ** 26, 0, kv_end=8)]
    assert _bytes(kv, over, L.DTYPE_F32)[0] == L.ERR_UNSUPPORTED and "too many rows" in _msg()
    assert _attend(kv, over, q, q) == L.ERR_UNSUPPORTED


def test_attend_kernel_modes():
    m, kv = _kv(pages=64, per_seq=64)
    L._call("laser_kv_add_seq", kv, 0, 1000)
    for mode in (-1, 3):
        assert _code("laser_model_set_attend_kernel", m, mode) == L.ERR_INVALID_ARG
    assert _code("laser_model_set_attend_kernel", None, 0) == L.ERR_STATE
    for mode in (0, 1, 2):
        L._call("laser_model_set_attend_kernel", m, mode)
        code, nb = _bytes(kv, [L.attend_span(0, 400, 600)])
        assert code == L.OK and nb % 4 == 0


def test_binding_passes_runs_and_spans_whole():
    runs = [L.kv_run(3, 5, 7, 9), L.kv_run(1, 0, 2)]
    data = L._joined(L.laser_kv_run, runs)
    assert list((C.c_int32 * 8).from_buffer_copy(data)) == [3, 5, 7, 9, 1, 0, 2, 0]
    assert bytes((L.laser_attend_span * 1)(L.attend_span(0, 4, 6))) == L._joined(L.laser_attend_span, (L.attend_span(0, 4, 6),))
    assert L._joined(L.laser_kv_run, []) == b""
    for bad in ([L.attend_span(0, 1, 0)], [(0, 1, 2, 3)], [1], [None]):
        with pytest.raises(TypeError):
            L._joined(L.laser_kv_run, bad)
