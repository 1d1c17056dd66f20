"""The operators where offsets pass 32 bits: the far end against the same operator on a slice of its own, or the formula."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2003_10579_amd import ssgd
    assert torch.cuda.is_available(), "this test needs the GPU"
    ssgd.lib()
    yield torch, ssgd
    torch.cuda.empty_cache()


def test_a_weight_of_more_than_4_gib(env):
    """300000 x 32768 in 4 bits: 4.9 GB of values, 0.3 GB of scales; one row, a few and a tile of them."""
    torch, ssgd = env
    N, K, tail = 300000, 32768, 100
    w = ssgd.MxTensor.empty(N, K, "fp4", torch.device("cuda", torch.cuda.current_device()))
    w.values.random_(0, 256)
    w.scales.random_(120, 130)
    end = ssgd.MxTensor(w.values[-tail:].contiguous(), w.scales[-tail:].contiguous(), "fp4", (tail, K))
    x = torch.randn(70, K, device="cuda").to(torch.bfloat16)
    for rows in (1, 20, 70):
        far, near = ssgd.mx_linear(x[:rows], w, "fp8", torch.float32)[:, -tail:], ssgd.mx_linear(x[:rows], end, "fp8", torch.float32)
        # (few rows of B and many may be added up in another order)
        assert torch.allclose(far, near, rtol=1e-4, atol=1e-4 * float(near.abs().max()))
    back = ssgd.mx_dequantize(end)
    assert torch.allclose(near[:1].double(), ssgd.mx_dequantize(ssgd.mx_quantize(x[:1], "fp8")).double() @ back.double().t(), rtol=1e-3,
                          atol=1e-4 * float(near.abs().max()))


def test_results_of_more_than_2_to_the_32(env):
    torch, ssgd = env
    n, k = 66000, 130
    a, b = ssgd.mx_quantize(torch.randn(n, k, device="cuda")), ssgd.mx_quantize(torch.randn(n, k, device="cuda"))
    out = ssgd.mx_matmul(a, b)
    assert out.numel() > 1 << 32
    cut = lambda q, rows: ssgd.MxTensor(q.values[rows].contiguous(), q.scales[rows].contiguous(), "fp4", (200, k))  # noqa: E731
    for rows in (slice(0, 200), slice(n - 200, n)):
        for cols in (slice(0, 200), slice(n - 200, n)):
            assert torch.equal(out[rows, cols], ssgd.mx_matmul(cut(a, rows), cut(b, cols)))


def test_quantisation_of_more_than_2_to_the_31(env):
    torch, ssgd = env
    rows, cols = 70000, 32768
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16).normal_()
    q, t = ssgd.mx_quantize_both(x, "fp8", "fp4")
    end = ssgd.mx_quantize(x[-64:], "fp8")
    assert torch.equal(q.values[-64:], end.values) and torch.equal(q.scales[-64:], end.scales)
    end = ssgd.mx_quantize_transposed(x[:, -64:], "fp4")
    assert torch.equal(t.values[-64:], end.values) and torch.equal(t.scales[-64:], end.scales)
    back = ssgd.mx_dequantize(q, torch.bfloat16)
    assert torch.equal(back[-64:], ssgd.mx_dequantize(ssgd.mx_quantize(x[-64:], "fp8"), torch.bfloat16))


def test_norm_of_more_than_2_to_the_31(env):
    torch, ssgd = env
    rows, d, tail = 270000, 8192, 50
    x = torch.empty(rows, d, device="cuda", dtype=torch.bfloat16).normal_()
    w = torch.ones(d, device="cuda")
    y, s, rstd = ssgd.rmsnorm(x, w, residual=x, output="fp8")
    y2, s2, rstd2 = ssgd.rmsnorm(x[-tail:], w, residual=x[-tail:], output="fp8")
    assert torch.equal(y.values[-tail:], y2.values) and torch.equal(s[-tail:], s2) and torch.equal(rstd[-tail:], rstd2)
    dx, dw = ssgd.rmsnorm_backward(x, s, w, rstd)
    dx2, _ = ssgd.rmsnorm_backward(x[-tail:], s2, w, rstd2)
    assert torch.equal(dx[-tail:], dx2) and torch.isfinite(dw).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_of_more_than_2_to_the_31(env, bits):
    torch, ssgd = env
    n, tail = (1 << 31) + 1001, 5000
    p = torch.zeros(n, device="cuda")
    g = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    g[:n // 2], g[n // 2:] = 0.5, -0.25
    opt = ssgd.AdamW([p[:7], p[7:]], state_bits=bits, weight_decay=0.0, max_norm=1e9)
    opt.step([g[:7], g[7:]], 0.125)
    # the first update is the rate times the gradient's sign, up to eps and the roundings of a handful of fp32 operations
    for part, sign in ((p[:tail], 1), (p[-tail:], -1)):
        assert torch.allclose(part, torch.full_like(part, -0.125 * sign), rtol=1e-6)
    norm = (n // 2 * 0.25 + (n - n // 2) * 0.0625) ** 0.5
    assert abs(float(opt.grad_norm) / norm - 1) < 1e-6
    at = 128 + n - 7 - tail          # the second tensor's place in the moments
    if bits == 32:
        assert torch.allclose(opt.m[at:at + tail], torch.full((tail,), -0.025, device="cuda"), rtol=1e-6)
    else:
        full = opt.m[at - at % 128:at + tail].float().view(-1)[:tail // 128 * 128]
        assert torch.all(full == -448) and torch.allclose(opt.m_scale[at // 128 + 1:at // 128 + 30], torch.full((29,), 0.025 / 448, device="cuda"), rtol=1e-6)
    opt.close()
