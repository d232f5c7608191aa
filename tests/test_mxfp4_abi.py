"""4-bit caches on the host: pool sizes, what models and pools are refused."""
import ctypes as C

import pytest

from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd.configs import QWEN_7B_FP4KV, ModelShape

PTR = 1 << 20  # an address that nothing reads


def _model(hd=64, dtype="bf16"):
    shape = ModelShape("abi", 2, 64, 4, 2, hd, 64, 64, True, False, dtype, 1.0e4, 1.0e-5, "mxfp4")
    desc, m = L.desc_from_shape(shape, 1024), C.c_void_p()
    return L.lib().laser_model_create(C.byref(desc), C.byref(m)), m


@pytest.mark.parametrize("hd", [64, 128])
def test_pool_bytes(hd):
    code, m = _model(hd)
    assert code == L.OK
    nb = C.c_size_t()
    L._call("laser_kv_pool_bytes", m, 10, C.byref(nb))
    assert nb.value == 2 * 10 * 2 * 16 * (hd // 2 + hd // 32)
    L._call("laser_model_destroy", m)


def test_needs_bf16_weights():
    assert _model(dtype="f32")[0] == L.ERR_UNSUPPORTED


def test_pools_are_aligned():
    _, m = _model()
    for k, v in ((PTR + 8, PTR), (PTR, PTR + 4)):
        out = C.c_void_p()
        assert L.lib().laser_kv_create(m, 4, 1, 4, k, v, PTR, C.byref(out)) == L.ERR_UNSUPPORTED
        assert "16-byte aligned" in L.lib().laser_last_error().decode()
    L._call("laser_model_destroy", m)


def test_bytes_per_token():
    s = QWEN_7B_FP4KV
    assert s.kv_bytes_per_token() == s.n_layers * 2 * s.n_kv_heads * 68
