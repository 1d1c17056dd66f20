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
    assert L.ssgd_adamw_state_elements(3, (C.c_int64 * 3)(*[1 << 47] * 3)) == -1


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


A = 0x1000       # an address that is never followed


def _refused(L, status, word):
    assert status == ssgd.EINVAL and word in L.ssgd_last_error(None)


def test_mx_row_bytes(L):
    for fmt, per in ((ssgd.MX_FP4, 2), (ssgd.MX_FP8, 1)):
        for cols, wide in ((0, 0), (1, 128), (128, 128), (129, 256), (3072, 3072)):
            assert L.ssgd_mx_row_bytes(fmt, cols) == wide // per
    assert L.ssgd_mx_row_bytes(2, 10) == -1 and L.ssgd_mx_row_bytes(0, -1) == -1 and L.ssgd_mx_row_bytes(0, 1 << 31) == -1


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=A + 2), dict(dtype=2), dict(rows=-1), dict(cols=-1), dict(pitch=99), dict(fmt=2), dict(fmt=-1), dict(values=None), dict(scales=None),
    dict(values=A + 8), dict(scales=A + 4), dict(values=None, scales=None), dict(fmt_t=2, values_t=A, scales_t=A), dict(values_t=A), dict(scales_t=A),
    dict(values_t=A + 8, scales_t=A), dict(cols=1 << 31, pitch=1 << 31), dict(rows=1 << 40), dict(rows=1 << 39), dict(rows=(1 << 40) - 1, cols=(1 << 31) - 1, pitch=1 << 31),
    dict(rows=1 << 34, cols=(1 << 30) + 1, pitch=1 << 31),
])
def test_mx_quantize_refuses(L, bad):
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_mx_quantize(g("x", A), g("dtype", 0), g("rows", 10), g("cols", 100), g("pitch", 100), g("fmt", 0), g("values", A), g("scales", A),
                                   g("fmt_t", 0), g("values_t", None), g("scales_t", None), None), b"mx")
    assert L.ssgd_mx_quantize(None, 0, 0, 100, 100, 0, None, None, 0, None, None, None) == ssgd.OK          # no rows: nothing to do


@pytest.mark.parametrize("bad", [dict(values=None), dict(scales=None), dict(out=None), dict(out=A + 2), dict(values=A + 4), dict(scales=A + 4), dict(fmt=2),
                                 dict(dtype=5), dict(rows=-1), dict(pitch=99), dict(rows=1 << 39), dict(rows=(1 << 40) - 1, cols=(1 << 31) - 1, pitch=1 << 31)])
def test_mx_dequantize_refuses(L, bad):
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_mx_dequantize(g("values", A), g("scales", A), g("fmt", 0), g("rows", 10), g("cols", 100), g("out", A), g("dtype", 0), g("pitch", 100), None), b"mx")


@pytest.mark.parametrize("bad", [dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(a=A + 8), dict(sa=A + 8), dict(b=A + 8), dict(sb=A + 8), dict(out=None),
                                 dict(out=A + 2), dict(fmt=2), dict(dtype=-1), dict(M=-1), dict(N=-1), dict(K=-1), dict(pitch=19), dict(M=1 << 31), dict(N=1 << 31, pitch=1 << 31),
                                 dict(K=1 << 24), dict(M=(1 << 31) - 1, N=(1 << 31) - 1, pitch=1 << 31)])
def test_mx_products_refuse(L, bad):
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_mx_matmul(g("a", A), g("sa", A), g("fmt", 0), g("M", 10), g("b", A), g("sb", A), g("N", 20), g("K", 100), g("out", A), g("dtype", 0), g("pitch", 20), A, None), b"mx")
    if not {"a", "sa"} & set(bad):
        for rows in (1, 10):
            M = g("M", rows)
            _refused(L, L.ssgd_mx_linear(A, 0, 1000, M, g("fmt", 0), g("b", A), g("sb", A), g("N", 20), g("K", 1000), g("out", A), g("dtype", 0), g("pitch", 20), A, None), b"mx")


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=A + 2), dict(kind=2), dict(pitch=999), dict(work=None), dict(work=A + 8)])
@pytest.mark.parametrize("rows", [1, 10])
def test_mx_linear_refuses(L, bad, rows):
    if rows == 1 and "work" in bad:
        assert L.ssgd_mx_linear_work_bytes(1, 1, 20, 1000) == 0            # one row needs none
        return
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_mx_linear(g("x", A), g("kind", 0), g("pitch", 1000), rows, 1, A, A, 20, 1000, A, 0, 20, g("work", A), None), b"mx")


def test_mx_work_bytes(L):
    linear, matmul = L.ssgd_mx_linear_work_bytes, L.ssgd_mx_matmul_work_bytes
    assert linear(1, 10, 50, 1000) == 10 * (1024 + 32) and linear(0, 9, 50, 1000) == 9 * (512 + 32)
    # a long contraction with few results is split, one with many or a short one is not; the parts are whole sets of results
    assert matmul(0, 128, 1000, 100000) >= 2 * 128 * 1000 * 4
    for fmt in (0, 1):
        for rows in (20, 64, 65, 128, 700):
            for n in (1000, 8192):
                for k in (4000, 8192, 30000):
                    parts = matmul(fmt, rows, n, k)
                    assert parts % (rows * n * 4) == 0 and parts <= 8 * rows * n * 4
                    wide = -(-k // 128) * 128
                    assert linear(fmt, rows, n, k) == parts + -(-rows * (wide // (1 if fmt else 2) + wide // 32) // 16) * 16
    assert matmul(0, 128, 8192, 128) == 0 and matmul(0, 8192, 8192, 8192) == 0 and matmul(1, 16, 8192, 8192) == 0 and matmul(1, 300, 300, 0) == 0
    for f in (linear, matmul):
        assert f(2, 10, 50, 1000) == -1 and f(0, -1, 50, 10) == -1 and f(0, 1, -1, 10) == -1 and f(0, 1, 50, 1 << 24) == -1
    _refused(L, L.ssgd_mx_matmul(A, A, 0, 128, A, A, 1000, 100000, A, 0, 1000, None, None), b"work")
    _refused(L, L.ssgd_mx_matmul(A, A, 0, 128, A, A, 1000, 100000, A, 0, 1000, A + 8, None), b"work")


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=A + 2), dict(w=None), dict(w=A + 1), dict(rstd=None), dict(dtype=2), dict(w_dtype=-1), dict(rows=-1), dict(d=0), dict(d=1 << 25, x_pitch=1 << 25, y_pitch=1 << 25), dict(x_pitch=99),
    dict(r=A), dict(sum=A), dict(r=A, sum=A, r_pitch=99), dict(r=A, sum=A, sum_pitch=99), dict(r=A + 2, sum=A), dict(y=None), dict(values=A, scales=A),
    dict(y=None, values=A), dict(y=None, values=A + 8, scales=A), dict(y=None, values=A, scales=A + 8), dict(y_pitch=99), dict(y=A + 2), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")),
])
def test_rmsnorm_refuses(L, bad):
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_rmsnorm(g("x", A), g("x_pitch", 100), g("r", None), g("r_pitch", 100), g("w", A), g("dtype", 0), g("w_dtype", 0), g("rows", 10), g("d", 100), g("eps", 1e-6),
                               g("sum", None), g("sum_pitch", 100), g("y", A), g("y_pitch", 100), g("values", None), g("scales", None), g("rstd", A), None), b"rmsnorm")


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(s=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(dy=A + 2), dict(dx=A + 2), dict(dtype=2), dict(w_dtype=2), dict(rows=-1), dict(d=0),
    dict(dy_pitch=99), dict(s_pitch=99), dict(dx_pitch=99), dict(dsum=A, dsum_pitch=99), dict(dsum=A + 2), dict(work=None), dict(work=A + 8), dict(dw=A + 2),
])
def test_rmsnorm_backward_refuses(L, bad):
    g = lambda k, d: bad.get(k, d)  # noqa: E731
    _refused(L, L.ssgd_rmsnorm_backward(g("dy", A), g("dy_pitch", 100), g("s", A), g("s_pitch", 100), g("w", A), g("dtype", 0), g("w_dtype", 0), g("rstd", A), g("dsum", None),
                                        g("dsum_pitch", 100), g("rows", 10), g("d", 100), g("dx", A), g("dx_pitch", 100), g("dw", A), g("work", A), None), b"rmsnorm")


def test_rmsnorm_work_floats(L):
    assert L.ssgd_rmsnorm_work_floats(0, 100) == 0
    for rows, d in ((1, 1), (3, 100), (1 << 20, 100), (1 << 20, 3000), (500, 20000)):       # a sum per workgroup
        floats = L.ssgd_rmsnorm_work_floats(rows, d)
        assert floats % d == 0 and 1 <= floats // d <= min(rows, 1024)
    assert L.ssgd_rmsnorm_work_floats(-1, 100) == -1 and L.ssgd_rmsnorm_work_floats(1, 0) == -1


@pytest.mark.parametrize("M,N,K", [(1, 1 << 28, 1000), (2, 1 << 27, 513), (1, 1 << 28, 100000), (16, 1 << 28, 1000), (10, (1 << 28) + 1, 640), (3, 1 << 29, 513)])
def test_mx_products_refuse_more_workgroups_than_a_launch_has(L, M, N, K):
    """Few rows of A and very many of B: a workgroup of 512 per 16 or 32 rows of B, and a launch has less than 2^32 threads."""
    _refused(L, L.ssgd_mx_linear(A, 0, K, M, 1, A, A, N, K, A, 0, N, A, None), b"too many")
    if N >= 1 << 28:
        _refused(L, L.ssgd_mx_matmul(A, A, 1, M, A, A, N, K, A, 0, N, A, None), b"too many")


@pytest.mark.parametrize("bad", [dict(eps=1e-50), dict(eps=1e39), dict(max_norm=1e-50)])
def test_adamw_refuses_what_fp32_does_not_hold(L, bad):
    """The update is in fp32: an eps or a norm to clip to that becomes zero there would divide by zero, or not clip at all."""
    o = ssgd.AdamWOptions(0.9, 0.999, bad.get("eps", 1e-8), bad.get("max_norm", 0.0), 32, 0)
    P, h = C.c_void_p * 1, C.c_void_p(0x1234)
    _refused(L, L.ssgd_adamw_create(1, (C.c_int64 * 1)(100), P(A), P(None), (C.c_double * 1)(0.1), C.byref(o), A, A, None, None, C.byref(h)), b"adamw")
    assert h.value == 0x1234
