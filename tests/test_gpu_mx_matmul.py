"""The product of microscaled matrices against the same values in 64 bits, through the public entry points."""
import numpy as np
import pytest

import mx_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2003_10579_amd import ssgd
    assert torch.cuda.is_available(), "this test needs the GPU"
    ssgd.lib()
    return torch, ssgd


def _host(x):
    return x.double().cpu().numpy()


def _matrix(torch, rows, cols, seed):
    """Every row at a level of its own, blocks of different sizes along it, a few large values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    x = x * torch.exp(1.5 * torch.randn(1, max(1, -(-cols // 32)), generator=g)).repeat_interleave(32, 1)[:, :cols]
    return x * (1 + 10 * (torch.rand(rows, cols, generator=g) < 0.01))


def _close(got, a, b, fmt, dtype):
    """a, b: the values that the operands stand for."""
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    steps = -(-a.shape[1] // 128)
    # one rounding of the running sum per 128 columns; 4 by 4 bits are exact within an instruction, of 8 by 4 bits it drops of each of 128
    # products what is below 2^-14 of the largest (a product of 2^-7 beside 448 and -448 is lost, one of 2^-5 is not)
    bound = (steps + 4) * 2.0 ** -24 * size + 1e-36
    if fmt == "fp8":
        for k in range(0, a.shape[1], 128):
            bound += 128 * 2.0 ** -14 * np.outer(np.abs(a[:, k:k + 128]).max(1), np.abs(b[:, k:k + 128]).max(1))
        assert np.linalg.norm(got - want) <= (1e-4 if dtype == "float32" else 2.0 ** -8) * np.linalg.norm(want)
    # then the rounding to the output's type
    place = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want) + bound, 1e-38))) - (24 if dtype == "float32" else 8))
    assert np.all(np.abs(got - want) <= bound + 1.01 * place)


# few rows (one, two and four groups of 16, partial ones), tiles of 64 and of 256; contractions from one column to
# many steps of 128, each remainder of the stages; rows of B that are no multiple of anything
SHAPES = [(1, 1, 1), (1, 3, 5), (2, 50, 900), (3, 50, 900), (2, 40, 17000), (1, 5200, 700), (16, 5130, 600), (20, 5121, 513), (50, 5150, 1300), (1, 16, 128), (1, 17, 4096), (1, 300, 3072), (2, 512, 3071), (15, 33, 129), (16, 100, 640), (17, 100, 512), (32, 40, 2200), (33, 70, 1000),
          (61, 130, 5000), (64, 64, 8192), (65, 1, 100), (65, 127, 300), (100, 129, 129), (65, 70, 5000), (128, 300, 9000), (200, 129, 3200), (256, 1000, 4225), (128, 128, 128), (129, 257, 256), (130, 130, 384), (300, 200, 512),
          (257, 513, 640), (512, 384, 1100), (3500, 3700, 127), (3585, 3600, 300), (3700, 3500, 700), (4000, 3500, 513)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_product(env, shape, fmt):
    torch, ssgd = env
    M, N, K = shape
    x, w = _matrix(torch, M, K, M + K), _matrix(torch, N, K, N + K + 1)
    a, b = ssgd.mx_quantize(x.cuda(), fmt), ssgd.mx_quantize(w.cuda(), "fp4")
    ah, bh = _host(ssgd.mx_dequantize(a)), _host(ssgd.mx_dequantize(b))
    if M * K < 1 << 20:
        assert np.array_equal(ah, ref.rounded(_host(x), fmt).astype(np.float32))
    for dtype in ("float32", "bfloat16"):
        out = ssgd.mx_matmul(a, b, getattr(torch, dtype))
        assert out.shape == (M, N) and out.dtype == getattr(torch, dtype)
        _close(_host(out), ah, bh, fmt, dtype)
    assert ssgd.mx_matmul(a, b).dtype == torch.bfloat16
    assert torch.equal(ssgd.mx_matmul(a, b), ssgd.mx_matmul(a, b))
    # the rows quantised on the way: the same bits
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype).cuda()
        assert torch.equal(ssgd.mx_linear(y, b, fmt), ssgd.mx_matmul(ssgd.mx_quantize(y, fmt), b, dtype))
    assert ssgd.mx_linear(x.cuda(), b, fmt, torch.bfloat16).dtype == torch.bfloat16


# tiles of 128, 96 and 64 rows with every kind of end, whole and in parts, 17 to 64 rows on either side of the rule between the kernels
TILES = [(2100, 1500, 900), (2050, 1030, 600), (1500, 1500, 1100), (1700, 1900, 2500), (900, 9000, 300), (1200, 1100, 600), (1000, 1000, 20000), (700, 700, 30000),
         (500, 500, 9000), (97, 260, 5000), (64, 512, 8200), (33, 6100, 8000), (24, 4100, 16000), (40, 28700, 130), (64, 16500, 700), (48, 51300, 300)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("shape", TILES, ids=str)
def test_product_by_tiles(env, shape, fmt):
    torch, ssgd = env
    M, N, K = shape
    x, w = _matrix(torch, M, K, M + K), _matrix(torch, N, K, N + K + 1)
    a, b = ssgd.mx_quantize(x.cuda(), fmt), ssgd.mx_quantize(w.cuda(), "fp4")
    ah, bh = _host(ssgd.mx_dequantize(a)), _host(ssgd.mx_dequantize(b))
    for dtype in ("float32", "bfloat16"):
        _close(_host(ssgd.mx_matmul(a, b, getattr(torch, dtype))), ah, bh, fmt, dtype)
    assert torch.equal(ssgd.mx_linear(x.cuda(), b, format=fmt), ssgd.mx_matmul(a, b, torch.float32))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_parts_of_every_length(env, fmt):
    """Contractions in parts whose last one has any number of steps, a single one too."""
    torch, ssgd = env
    for K in range(1900, 6000, 128):
        x, w = _matrix(torch, 65, K, K), _matrix(torch, 130, K, K + 1)
        a, b = ssgd.mx_quantize(x.cuda(), fmt), ssgd.mx_quantize(w.cuda(), "fp4")
        _close(_host(ssgd.mx_matmul(a, b, torch.float32)), _host(ssgd.mx_dequantize(a)), _host(ssgd.mx_dequantize(b)), fmt, "float32")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_a_layer_forward_and_backward(env, fmt):
    """y = x w^T, dx = dy w, dw = dy^T x by quantisation along rows and columns: each against the product of the values that its own
    operands stand for."""
    torch, ssgd = env
    T, N, K = 200, 96, 160
    x, w, dy = (_matrix(torch, *s, k).cuda() for k, s in enumerate(((T, K), (N, K), (T, N))))
    (xq, xt), (wq, wt), (dq, dt) = ssgd.mx_quantize_both(x, fmt, "fp4"), ssgd.mx_quantize_both(w, "fp4", "fp4"), ssgd.mx_quantize_both(dy, fmt, fmt)
    for a, b, left, right in ((xq, wq, x, w), (dq, wt, dy, w.t()), (dt, xt, dy.t(), x.t())):
        got = _host(ssgd.mx_matmul(a, b, torch.float32))
        _close(got, ref.rounded(_host(left), a.format), ref.rounded(_host(right), "fp4"), a.format, "float32")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_gradients_of_a_layer_against_differences(env, fmt):
    """With values that both formats hold exactly along rows and columns, the layer is the unquantised one: its gradients against central
    differences of sum(dy * y), which are exact for a function linear in each argument, up to the rounding of the differences."""
    torch, ssgd = env
    T, N, K = 70, 40, 100
    g = torch.Generator().manual_seed(4)
    pick = lambda *s: torch.tensor(ref.TABLE["fp4"], dtype=torch.float32)[torch.randint(1, 8, s, generator=g)] * torch.randint(0, 2, s, generator=g).mul(2).sub(1)  # noqa: E731
    x, w, dy = pick(T, K), pick(N, K), pick(T, N)
    (xq, xt), (wq, wt), (dq, dt) = (ssgd.mx_quantize_both(t.cuda(), f, h) for t, f, h in ((x, fmt, "fp4"), (w, "fp4", "fp4"), (dy, fmt, fmt)))
    y, dx, dw = (_host(ssgd.mx_matmul(a, b, torch.float32)) for a, b in ((xq, wq), (dq, wt), (dt, xt)))
    xh, wh, dyh = _host(x), _host(w), _host(dy)
    assert np.array_equal(y, xh @ wh.T)
    for i, k in ((0, 0), (33, 99), (69, 50)):
        e = np.zeros_like(xh); e[i, k] = 0.5
        assert abs((dyh * ((xh + e) @ wh.T)).sum() - (dyh * ((xh - e) @ wh.T)).sum() - dx[i, k]) < 1e-9
    for n, k in ((0, 0), (20, 99), (39, 31)):
        e = np.zeros_like(wh); e[n, k] = 0.5
        assert abs((dyh * (xh @ (wh + e).T)).sum() - (dyh * (xh @ (wh - e).T)).sum() - dw[n, k]) < 1e-9


def test_blocks_that_are_nan_and_large_scales(env):
    torch, ssgd = env
    for M, N in ((3, 40), (100, 140), (3600, 3600)):
        x, w = torch.ones(M, 300), torch.ones(N, 300)
        x[1, 40] = float("inf")
        w[5, 299] = float("nan")
        for fmt in ("fp4", "fp8"):
            out = ssgd.mx_linear(x.cuda(), ssgd.mx_quantize(w.cuda(), "fp4"), fmt).cpu()
            assert torch.isnan(out[1]).all() and torch.isnan(out[:, 5]).all()
            out[1], out[:, 5] = 300, 300
            assert torch.all(out == 300)
    # 2^120 times 2^-120, 2^100 times 2^100: finite, and past the range
    one = torch.ones(70, 128, device="cuda")
    small, large = ssgd.mx_quantize(one * 2.0 ** -120), ssgd.mx_quantize(one * 2.0 ** 120)
    assert torch.all(ssgd.mx_matmul(small, large, torch.float32) == 128)
    huge = ssgd.mx_quantize(one * 2.0 ** 100)
    assert torch.isinf(ssgd.mx_matmul(huge, huge, torch.float32)).all()


def test_strided_and_misaligned_outputs_and_nothing_beside_them(env):
    """Through the C entry, with room around the rows of the output."""
    torch, ssgd = env
    L = ssgd.lib()
    stream = torch.cuda.current_stream().cuda_stream
    for M, N, K in ((1, 37, 200), (50, 130, 700), (140, 135, 300), (140, 135, 5000), (3500, 3601, 130)):
        a, b = ssgd.mx_quantize(_matrix(torch, M, K, 1).cuda(), "fp8"), ssgd.mx_quantize(_matrix(torch, N, K, 2).cuda(), "fp4")
        want = ssgd.mx_matmul(a, b, torch.float32)
        work = torch.full((L.ssgd_mx_matmul_work_bytes(1, M, N, K) // 4 + 8,), float("nan"), device="cuda")
        for pad, offset in ((0, 0), (8, 4), (5, 1)):
            room = torch.full((M + 2, N + pad), 7.0, device="cuda")
            assert L.ssgd_mx_matmul(a.values.data_ptr(), a.scales.data_ptr(), 1, M, b.values.data_ptr(), b.scales.data_ptr(), N, K,
                                    room[1:].data_ptr() + 4 * offset, 0, N + pad, work.data_ptr(), stream) == 0
            flat = room.reshape(-1)
            at = N + pad + offset
            body = flat[at:at + (M - 1) * (N + pad) + N]
            got = torch.stack([body[i * (N + pad):i * (N + pad) + N] for i in (0, M // 2, M - 1)])
            assert torch.equal(got, want[[0, M // 2, M - 1]])
            assert torch.all(flat[:at] == 7) and torch.all(flat[at + (M - 1) * (N + pad) + N:] == 7)
            assert torch.all(torch.as_strided(flat, (M - 1, pad), (N + pad, 1), at + N) == 7)      # between the rows


def test_empty_products(env):
    torch, ssgd = env
    e = lambda r, c, f="fp4": ssgd.mx_quantize(torch.zeros(r, c, device="cuda"), f)  # noqa: E731
    assert ssgd.mx_matmul(e(0, 64), e(5, 64)).shape == (0, 5) and ssgd.mx_matmul(e(5, 64), e(0, 64)).shape == (5, 0)
    for dtype in (torch.float32, torch.bfloat16):
        out = ssgd.mx_matmul(e(70, 0), e(90, 0), dtype)
        assert out.shape == (70, 90) and torch.all(out == 0)
        assert torch.all(ssgd.mx_linear(torch.zeros(3, 0, device="cuda", dtype=dtype), e(4, 0)) == 0)
    assert ssgd.mx_linear(torch.zeros(0, 64, device="cuda"), e(4, 64)).shape == (0, 4)


def test_another_stream_and_a_replayed_graph_give_the_same(env):
    torch, ssgd = env
    x, w = _matrix(torch, 90, 9000, 1).cuda().bfloat16(), ssgd.mx_quantize(_matrix(torch, 333, 9000, 2).cuda(), "fp4")
    for rows in (1, 90):          # (90 rows: quantised, split and joined)
        want = ssgd.mx_linear(x[:rows], w)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got = ssgd.mx_linear(x[:rows], w)
        s.synchronize()
        assert torch.equal(want, got)
        graph = torch.cuda.CUDAGraph()
        y = x[:rows].clone()
        with torch.cuda.graph(graph):
            out = ssgd.mx_linear(y, w)
        for k in range(3):
            y.copy_(x[:rows] * (k + 1))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ssgd.mx_linear(y, w))


def test_refusals(env):
    torch, ssgd = env
    x = torch.zeros(4, 64, device="cuda")
    a, b, f8 = ssgd.mx_quantize(x), ssgd.mx_quantize(torch.zeros(6, 64, device="cuda")), ssgd.mx_quantize(x, "fp8")
    other = ssgd.mx_quantize(torch.zeros(6, 65, device="cuda"))
    for call in (lambda: ssgd.mx_matmul(a, f8), lambda: ssgd.mx_matmul(a, other), lambda: ssgd.mx_matmul(x, b), lambda: ssgd.mx_matmul(a, x),
                 lambda: ssgd.mx_matmul(a, b, torch.float16), lambda: ssgd.mx_linear(x, f8), lambda: ssgd.mx_linear(x, other), lambda: ssgd.mx_linear(x, b, "int8"),
                 lambda: ssgd.mx_linear(x.half(), b), lambda: ssgd.mx_linear(x.cpu(), b), lambda: ssgd.mx_linear(x, b, "fp8", torch.float64), lambda: ssgd.mx_linear(x.t(), b)):
        with pytest.raises(ssgd.SsgdError) as e:
            call()
        assert e.value.status == ssgd.EINVAL


def test_stored_matrices_in_a_first_call(env, monkeypatch):
    """A product, and values read back, of matrices from stored arrays before any other operator has run."""
    torch, ssgd = env
    a, b = (ssgd.mx_quantize(_matrix(torch, n, 300, n).cuda(), f) for n, f in ((5, "fp8"), (9, "fp4")))
    want, back = ssgd.mx_matmul(a, b, torch.float32), ssgd.mx_dequantize(a, torch.bfloat16)
    arrays = [(q.values, q.scales, q.format, q.shape) for q in (a, b)]
    def fresh():
        for name in ("_torch", "_raw_stream", "_device_now"):
            monkeypatch.setattr(ssgd, name, None)
        monkeypatch.setattr(ssgd, "_DTYPES", {})
        return [ssgd.MxTensor(*q) for q in arrays]
    assert torch.equal(ssgd.mx_matmul(*fresh(), torch.float32), want)
    assert torch.equal(ssgd.mx_dequantize(fresh()[0], torch.bfloat16), back)


def _cut(torch, x, offset, pad):
    """The same rows inside wider ones of NaN."""
    room = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device="cuda")
    room[:, offset:offset + x.shape[1]] = x
    return room[:, offset:offset + x.shape[1]]


def _same(torch, a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=7.0), torch.nan_to_num(b, nan=7.0))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("K", [513, 519, 544, 640, 2999, 8191])
def test_one_and_two_rows_from_any_place_and_with_any_values(env, K, fmt, dtype):
    """The product that quantises its rows itself: rows at odd places among NaN, blocks with infinities and NaN (the first, one inside, the last), of zeros,
    of the smallest and the largest numbers, as quantisation and product one after the other have them."""
    torch, ssgd = env
    dt, N = getattr(torch, dtype), 70
    b = ssgd.mx_quantize(_matrix(torch, N, K, 2).cuda(), "fp4")
    for M in (1, 2):
        x = _matrix(torch, M, K, K + M).to(dt).cuda()
        special = []
        for at in (0, K // 2, K - 1):
            for value in (float("inf"), -float("inf"), float("nan")):
                y = x.clone()
                y[-1, at] = value
                special.append(y)
        y = x.clone(); y[0, :300] = 0.0; special.append(y)
        special += [torch.zeros_like(x), x * 1e-38, x.sign() * 3e38, x * 2.0 ** -133]
        for y in [x] + special:
            want = ssgd.mx_matmul(ssgd.mx_quantize(y, fmt), b, torch.float32)
            assert _same(torch, ssgd.mx_linear(y, b, fmt, torch.float32), want)
            for offset, pad in ((1, 3), (3, 7), (8, 8)):
                assert _same(torch, ssgd.mx_linear(_cut(torch, y, offset, pad), b, fmt, torch.float32), want)
        assert all(torch.isnan(ssgd.mx_linear(y, b, fmt)[-1]).all() for y in special[:9])
        if M == 2:
            assert not any(torch.isnan(ssgd.mx_linear(y, b, fmt)[0]).any() for y in special[:9])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M", [3, 16, 17, 40, 64, 70, 300])
def test_rows_from_any_place(env, M, fmt):
    torch, ssgd = env
    for N, K in ((70, 200), (5200, 700), (300, 5000)):
        b, x = ssgd.mx_quantize(_matrix(torch, N, K, 2).cuda(), "fp4"), _matrix(torch, M, K, 3).cuda()
        for dt in (torch.float32, torch.bfloat16):
            y = x.to(dt)
            want = ssgd.mx_matmul(ssgd.mx_quantize(y, fmt), b, dt)
            for offset, pad in ((1, 3), (3, 7), (8, 8)):
                assert torch.equal(ssgd.mx_linear(_cut(torch, y, offset, pad), b, fmt), want)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kind", [0, 1])
def test_strided_and_misaligned_outputs_whole(env, fmt, kind):
    """Every row of an output whose rows lie apart and begin anywhere, in both types, through the C entries of the product and of the layer."""
    torch, ssgd = env
    L, dt, name = ssgd.lib(), (torch.float32, torch.bfloat16)[kind], ("fp4", "fp8")[fmt]
    stream = torch.cuda.current_stream().cuda_stream
    for M, N, K in ((1, 37, 200), (1, 37, 700), (2, 5125, 700), (16, 130, 700), (30, 5201, 700), (50, 130, 700), (64, 5201, 1300), (140, 135, 300), (140, 135, 5000), (300, 517, 900),
                    (1100, 1205, 300), (3500, 3601, 130)):
        x = _matrix(torch, M, K, 1).cuda()
        a, b = ssgd.mx_quantize(x, name), ssgd.mx_quantize(_matrix(torch, N, K, 2).cuda(), "fp4")
        want = ssgd.mx_matmul(a, b, dt)
        work = torch.full((max(L.ssgd_mx_matmul_work_bytes(fmt, M, N, K), L.ssgd_mx_linear_work_bytes(fmt, M, N, K)) // 4 + 8,), float("nan"), device="cuda")
        for pad, offset in ((0, 0), (8, 4), (5, 1), (3, 2)):
            for layer in (False, True):
                room = torch.full((M + 2, N + pad), 7.0, device="cuda", dtype=dt)
                flat, at = room.reshape(-1), N + pad + offset
                out = flat.data_ptr() + at * flat.element_size()
                if layer:
                    status = L.ssgd_mx_linear(x.data_ptr(), 0, K, M, fmt, b.values.data_ptr(), b.scales.data_ptr(), N, K, out, kind, N + pad, work.data_ptr(), stream)
                else:
                    status = L.ssgd_mx_matmul(a.values.data_ptr(), a.scales.data_ptr(), fmt, M, b.values.data_ptr(), b.scales.data_ptr(), N, K, out, kind, N + pad, work.data_ptr(), stream)
                assert status == 0
                body = torch.as_strided(flat, (M, N), (N + pad, 1), at)
                assert torch.equal(body, want), (M, N, K, pad, offset, layer)
                body.fill_(7.0)
                assert torch.all(flat == 7)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_the_smallest_and_largest_scales(env, fmt):
    """Blocks with scale byte 0 (2^-127, from numbers at and below the smallest normal ones) and with the largest one, through every kernel."""
    torch, ssgd = env
    for M, N, K in ((1, 40, 256), (1, 40, 1024), (2, 40, 640), (20, 40, 640), (70, 140, 640), (300, 517, 640)):
        one, other = torch.ones(M, K, device="cuda"), torch.ones(N, K, device="cuda")
        for low, high in ((-126, 120), (-128, 125), (-128, 127), (-127, 60)):        # (half of 2^-127 is the smallest E2M1 has)
            small, large = one * 2.0 ** -100 * 2.0 ** (low + 100), ssgd.mx_quantize(other * 2.0 ** high)
            assert torch.all(small > 0)
            want = torch.full((M, N), K * 2.0 ** (low + high), device="cuda")
            q = ssgd.mx_quantize(small, fmt)
            assert torch.equal(ssgd.mx_matmul(q, large, torch.float32), want) and torch.equal(ssgd.mx_linear(small, large, fmt), want)
            assert torch.equal(ssgd.mx_matmul(ssgd.mx_quantize(one * 2.0 ** high, fmt), ssgd.mx_quantize(other * 2.0 ** -100 * 2.0 ** (low + 100)), torch.float32), want)
