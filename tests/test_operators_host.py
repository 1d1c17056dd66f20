"""Host-side checks of the operators that need no GPU: invalid arguments are refused before the device is touched."""
import ctypes as C
import os

import pytest

from paper_2003_10579_amd import ssgd


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ssgd._LIB_PATH):
        from paper_2003_10579_amd import build
        build.build()
    return ssgd.lib()


def test_adamw_state_elements(L):
    sizes = (C.c_int64 * 5)(1, 128, 129, 0, 3072 * 512)
    assert L.ssgd_adamw_state_elements(5, sizes) == 128 + 128 + 256 + 3072 * 512
    assert L.ssgd_adamw_state_elements(0, sizes) == -1
    assert L.ssgd_adamw_state_elements(1, None) == -1
    assert L.ssgd_adamw_state_elements(1, (C.c_int64 * 1)(-1)) == -1


@pytest.mark.parametrize("bad", [
    dict(tensors=0), dict(sizes=-1), dict(params=None), dict(param=None), dict(param=0x1001), dict(copy=0x1001), dict(decay=float("nan")),
    dict(decay=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=float("inf")),
    dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(bits=16), dict(m=None), dict(v=None), dict(m=0x1004), dict(v=0x1008),
    dict(bits=8, m_scale=None), dict(bits=8, v_scale=None), dict(sizes=1 << 45),
])
def test_adamw_create_refuses(L, bad):
    o = ssgd.AdamWOptions(bad.get("beta1", 0.9), bad.get("beta2", 0.999), bad.get("eps", 1e-8), bad.get("max_norm", 0.0), bad.get("bits", 32), 0)
    P = C.c_void_p * 1
    params = None if "params" in bad else P(bad.get("param", 0x1000))
    h = C.c_void_p(0x1234)
    st = L.ssgd_adamw_create(bad.get("tensors", 1), (C.c_int64 * 1)(bad.get("sizes", 100)), params, P(bad.get("copy", None)),
                             (C.c_double * 1)(bad.get("decay", 0.1)), C.byref(o), bad.get("m", 0x1000), bad.get("v", 0x1000),
                             bad.get("m_scale", 0x1000), bad.get("v_scale", 0x1000), C.byref(h))
    assert st == ssgd.EINVAL and b"adamw" in L.ssgd_last_error(None)
    assert h.value == 0x1234


def test_adamw_null_handle(L):
    grads = (C.c_void_p * 1)(0x1000)
    assert L.ssgd_adamw_step(None, grads, ssgd.F32, 0.1, 1, None, None) == ssgd.EINVAL
    L.ssgd_adamw_destroy(None)
