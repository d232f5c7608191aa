"""Rotary positions on the host: the scaled frequencies against their formulas, and what laser_rotate and
laser_kv_write_rotated refuse, over pointers that are never followed."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd.configs import ModelShape

PTR = 1 << 20


def _freq(rot, theta, *scaling):
    return L.laser_rope_frequencies(rot, theta, L.laser_rope_scaling(*scaling) if scaling else None)


@pytest.mark.parametrize("rot,theta", [(2, 1.0e4), (4, 1.0e4), (30, 1.0e4), (64, 5.0e5), (128, 1.0e4), (128, 1.0e6)])
def test_frequencies(rot, theta):
    i = np.arange(rot // 2)
    f = theta ** (-2.0 * i / rot)
    close = lambda got, ref: np.allclose(got, ref, rtol=1e-13, atol=0)  # noqa: E731
    got, a = _freq(rot, theta)
    assert a == 1.0 and close(got, f) and got[0] == 1.0
    got, a = _freq(rot, theta, 1, 4.0, 0.0, 0.0, 0.0)
    assert a == 1.0 and close(got, f / 4)
    got, a = _freq(rot, theta, 2, 4.0, 0.0, 0.0, 0.0)
    assert a == 1.0 and close(got[0], 1.0)
    if rot > 2:  # the slowest pair is 4 times slower
        assert close(got[-1], f[-1] / 4)
    got, a = _freq(rot, theta, 3, 8.0, 8192.0, 1.0, 4.0)
    for x, y in zip(got, f):
        turns = 8192.0 * y / (2 * math.pi)
        ref = y if turns >= 4 else y / 8 if turns <= 1 else y * ((turns - 1) / 3 + (4 - turns) / 3 / 8)
        assert close(x, ref)
    got, a = _freq(rot, theta, 4, 4.0, 4096.0, 1.0, 32.0)
    assert close(a, 1 + 0.1 * math.log(4.0))
    lo, hi = (rot * math.log(4096.0 / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (32.0, 1.0))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
    for j, (x, y) in enumerate(zip(got, f)):
        r = min(1.0, max(0.0, (j - lo) / max(hi - lo, 1e-3)))
        assert close(x, y * (1 - r) + y / 4 * r)


def test_frequencies_refused():
    bad = [(0, 1e4), (3, 1e4), (-2, 1e4), (8, 1.0), (8, -5.0), (8, math.inf), (8, math.nan)]
    for rot, theta in bad:
        with pytest.raises(L.LaserError):
            _freq(rot, theta)
    for s in ((9, 2.0, 1.0, 1.0, 2.0), (-1, 2.0, 1.0, 1.0, 2.0), (1, 0.0, 1.0, 1.0, 2.0), (2, -1.0, 1.0, 1.0, 2.0), (1, math.nan, 1.0, 1.0, 2.0),
              (3, 2.0, 0.0, 1.0, 2.0), (3, 2.0, 10.0, 0.0, 2.0), (3, 2.0, 10.0, 2.0, 2.0), (4, 0.5, 10.0, 1.0, 2.0), (4, 2.0, 10.0, 1.0, math.inf)):
        with pytest.raises(L.LaserError) as e:
            _freq(8, 1e4, *s)
        assert e.value.code == L.ERR_INVALID_ARG
    assert L.lib().laser_rope_frequencies(8, 1e4, None, None, None) == L.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        L.rope(64, layout="other")
    with pytest.raises(ValueError):
        L.rope(64, scaling="other")
    with pytest.raises(ValueError):
        L.rope(64, inv_freq=[1.0] * 31)


def test_frequencies_beyond_double():
    """A factor that leaves the doubles' range is refused, and nothing is written."""
    for rot, theta, s in ((4, 1e4, (2, 1e200, 0.0, 0.0, 0.0)), (4, 1e4, (2, 1e-200, 0.0, 0.0, 0.0)), (64, 1e4, (1, 5e-324, 0.0, 0.0, 0.0)),
                          (64, 1e4, (3, 5e-324, 1.0, 1.0, 4.0))):
        f, a = (C.c_double * (rot // 2))(*[-1.0] * (rot // 2)), C.c_double(-1.0)
        sc = L.laser_rope_scaling(*s)
        assert L.lib().laser_rope_frequencies(rot, theta, C.byref(sc), f, C.byref(a)) == L.ERR_INVALID_ARG
        assert list(f) == [-1.0] * (rot // 2) and a.value == -1.0
    with pytest.raises(ValueError):
        L.rope(64, scaling="linear", factor=2.0, inv_freq=[1.0] * 32)


def _rows(n, heads, dtype=L.DTYPE_BF16, ptr=PTR, row=None, head=64):
    return L.laser_rows(ptr, dtype, n, heads * 64 if row is None else row, head)


def _rotate(rope, runs, x, out, heads=4):
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return L.lib().laser_rotate(ref(rope), len(runs), L._joined(L.laser_rotate_run, runs), heads, ref(x), ref(out), None)


def test_rotate_refused():
    rope, x, out = L.rope(64), _rows(10, 4), _rows(10, 4, ptr=2 * PTR)
    R = L.rotate_run
    inv, uns = L.ERR_INVALID_ARG, L.ERR_UNSUPPORTED
    assert _rotate(rope, [], x, out) == L.OK and _rotate(rope, [R(0, 5), R(0, 3, 10)], x, out) == L.OK
    for runs in ([R(-1, 0)], [R(11, 0)], [R(1, 0, 10)], [R(1, 0, -1)], [R(2, 0), R(1, 0, 1)], [R(1, 0), R(1, 9)], [R(2 ** 31 - 1, 0, 1)]):
        assert _rotate(rope, runs, x, out) == inv, runs
    one = [R(1, 0)]
    assert _rotate(None, one, x, out) == inv and _rotate(rope, one, None, out) == inv and _rotate(rope, one, x, None) == inv
    assert L.lib().laser_rotate(C.byref(rope), 1, None, 4, C.byref(x), C.byref(out), None) == inv
    assert _rotate(rope, one, x, out, 0) == inv and _rotate(rope, one, x, out, -1) == inv and _rotate(rope, one, x, out, 8193) == uns
    assert _rotate(rope, one, x, _rows(10, 4, L.DTYPE_F32)) == uns
    assert _rotate(rope, one, _rows(10, 4, L.DTYPE_INT8), _rows(10, 4, L.DTYPE_INT8)) == uns
    assert _rotate(rope, one, x, _rows(10, 4, row=200)) == inv  # written rows overlap
    assert _rotate(rope, one, x, _rows(10, 4, row=512)) == inv  # x's own memory, other strides
    assert _rotate(rope, one, _rows(10, 4, ptr=PTR + 1), out) == inv
    assert _rotate(rope, one, _rows(10, 4, row=-1), out) == inv
    for r, code in ((L.rope(64, rot_dim=32), None), (L.laser_rope(64, 33, 0, 1.0, rope.inv_freq), inv), (L.laser_rope(64, 66, 0, 1.0, rope.inv_freq), inv),
                    (L.laser_rope(64, 0, 0, 1.0, rope.inv_freq), inv), (L.laser_rope(64, 64, 2, 1.0, rope.inv_freq), inv),
                    (L.laser_rope(64, 64, 0, math.nan, rope.inv_freq), inv), (L.laser_rope(64, 64, 0, 1.0, None), inv),
                    (L.laser_rope(258, 64, 0, 1.0, rope.inv_freq), uns), (L.laser_rope(0, 64, 0, 1.0, rope.inv_freq), uns),
                    (L.rope(64, inv_freq=[1.0] * 31 + [math.inf]), inv), (L.rope(64, inv_freq=[math.nan] + [1.0] * 31), inv),
                    (L.rope(64, inv_freq=[2.0 ** 20] * 32), inv)):
        assert _rotate(r, [], x, out) == (L.OK if code is None else code)


def _kv(kind):
    shape = ModelShape("abi", 2, 64, 4, 2, 64, 64, 64, True, False, "f32" if kind == "f32" else "bf16", 1.0e4, 1.0e-5,
                       kind if kind in ("fp8", "int8", "mxfp4") else "")
    desc = L.desc_from_shape(shape, 1024)
    m, kv = C.c_void_p(), C.c_void_p()
    L._call("laser_model_create", C.byref(desc), C.byref(m))
    L._call("laser_kv_create", m, 64, 4, 32, PTR, PTR + (1 << 24), PTR + (1 << 25), C.byref(kv))
    return m, kv


@pytest.mark.parametrize("kind", ["mxfp4", "int8", "fp8", "bf16", "f32"])
def test_write_rotated_refused(kind):
    """A call whose arguments are in order ends with STATE: the model is not finalized."""
    _, kv = _kv(kind)
    L._call("laser_kv_add_seq", kv, 0, 40)
    L._call("laser_kv_add_seq", kv, 1, 16)
    rope = L.rope(64)
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731

    def call(runs, k=_rows(50, 2), v=_rows(50, 2, ptr=3 * PTR), q=None, q_out=None, r=rope, layer=0, handle=kv):
        return L.lib().laser_kv_write_rotated(handle, layer, ref(r), len(runs), L._joined(L.laser_kv_run, runs), ref(k), ref(v), ref(q),
                                              ref(q_out), None)

    inv, uns, state = L.ERR_INVALID_ARG, L.ERR_UNSUPPORTED, L.ERR_STATE
    ok = [L.kv_run(0, 3, 20), L.kv_run(1, 0, 16, 20)]
    q, qo = _rows(50, 4, ptr=5 * PTR), _rows(50, 4, ptr=6 * PTR)
    assert call(ok) == state and call(ok, q=q, q_out=qo) == state and call(ok, q=q, q_out=q) == state
    assert call([], None, None) == state
    assert call(ok, r=None) == inv and call(ok, r=L.rope(128)) == inv and call(ok, r=L.laser_rope(64, 3, 0, 1.0, rope.inv_freq)) == inv
    assert call(ok, q=q) == inv and call(ok, q_out=qo) == inv
    assert call(ok, q=_rows(50, 4, L.DTYPE_F32), q_out=_rows(50, 4, L.DTYPE_F32, 6 * PTR)) == uns
    assert call(ok, q=q, q_out=_rows(50, 4, ptr=6 * PTR, row=100)) == inv
    assert call(ok, q=q, q_out=_rows(50, 4, ptr=5 * PTR, row=512)) == inv
    assert call(ok, q=_rows(30, 4, ptr=5 * PTR), q_out=qo) == inv and call(ok, q=q, q_out=_rows(30, 4, ptr=6 * PTR)) == inv
    both = [L.kv_run(0, 3, 16, 20), L.kv_run(1, 0, 16, 20)]  # the same rows into two sequences: with queries each of theirs once
    assert call(both) == state and call(both, q=q, q_out=qo) == inv
    assert call([L.kv_run(0, 30, 11)]) == inv and call([L.kv_run(2, 0, 1)]) == inv and call([L.kv_run(0, 0, 2), L.kv_run(0, 1, 1)]) == inv
    assert call(ok, layer=2) == inv and call(ok, handle=None) == state
    assert call(ok, k=_rows(50, 2, L.DTYPE_F32)) == uns and call(ok, k=None) == inv


def test_set_rope_refused():
    m, _ = _kv("bf16")
    call = lambda h, r: L.lib().laser_model_set_rope(h, None if r is None else C.byref(r))  # noqa: E731
    assert call(m, L.rope(64, 5.0e5, scaling="linear", factor=2.0)) == L.OK and call(m, L.rope(64)) == L.OK
    assert call(None, L.rope(64)) == L.ERR_STATE
    assert call(m, None) == L.ERR_INVALID_ARG and call(m, L.rope(128)) == L.ERR_INVALID_ARG
    assert call(m, L.rope(64, rot_dim=32)) == L.ERR_UNSUPPORTED and call(m, L.rope(64, layout="interleaved")) == L.ERR_UNSUPPORTED


def test_q_out_is_not_k_or_v():
    _, kv = _kv("mxfp4")
    L._call("laser_kv_add_seq", kv, 0, 40)
    rope, q = L.rope(64), _rows(50, 4, ptr=5 * PTR)
    runs = L._joined(L.laser_kv_run, [L.kv_run(0, 3, 20)])
    for at, code in ((PTR, L.ERR_INVALID_ARG), (3 * PTR, L.ERR_INVALID_ARG), (6 * PTR, L.ERR_STATE)):
        k, v, out = _rows(50, 2), _rows(50, 2, ptr=3 * PTR), _rows(50, 4, ptr=at)
        assert L.lib().laser_kv_write_rotated(kv, 0, C.byref(rope), 1, runs, C.byref(k), C.byref(v), C.byref(q), C.byref(out), None) == code
