"""The product with a dense layer's or a gated block's epilogue against the same values in 64 bits, through the public entry points."""
import math

import numpy as np
import pytest

import mx_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24          # half a unit in the last place of fp32, relative


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
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g))
    return x * (1 + 10 * (torch.rand(rows, cols, generator=g) < 0.01))


def _act(x, name):
    from scipy.special import expit, ndtr
    return {None: lambda: x, "relu": lambda: np.maximum(x, 0), "gelu": lambda: x * ndtr(x), "silu": lambda: x * expit(x)}[name]()


def _act_error(x, name):
    """What the kernel's own evaluation may be off by: relu is exact; silu's exponent is rounded (|x| half units), then an exponential, a quotient, a sum and a
    product of at most two units each, and where 1 + e^-x is past 2^126 its quotient is below fp32's normal numbers, or e^-x past its range, and counts as zero: that is
    for x < -126 ln 2 = -87.3, where |x| / (1 + e^-x) < 88 x 2^-126 and falls; Phi has 3.4e-9 and the rounding of x^2 / 2 in its exponent, and eight roundings behind it, at most one in full."""
    if name == "silu":
        return np.abs(_act(x, name)) * (2 * np.abs(x) + 12) * U + np.where(x < -87.0, 88 * 2.0 ** -126, 0.0)
    if name == "gelu":
        bell = np.exp(-x * x / 2)
        return np.abs(x) * (3.4e-9 + bell * (2 * x * x + 24) * U / 2 + 2 * U) + np.abs(_act(x, name)) * 2 * U + 1e-37
    return np.zeros_like(x)


def _sums(a, b, fmt):
    """p and its bound: one rounding of the running sum per 128 columns, and what the unit drops of 8 by 4 bits (2^-14 of the largest of 128 products, of each)."""
    p, size = a @ b.T, np.abs(a) @ np.abs(b).T
    bound = (-(-a.shape[1] // 128) + 4) * U * size + 1e-36
    if fmt == "fp8":
        for k in range(0, a.shape[1], 128):
            bound += 128 * 2.0 ** -14 * np.outer(np.abs(a[:, k:k + 128]).max(1), np.abs(b[:, k:k + 128]).max(1))
    return p, bound


def _within(got, want, bound):
    assert got.shape == want.shape and np.all(np.abs(got - want) <= bound + 2 * U * np.abs(want))


# few rows quantised on the way, few rows, 17 to 64 of them, tiles of 64, 96, 128 and 256, contractions in parts and of no columns, odd sizes
SHAPES = [(1, 1, 1), (1, 70, 900), (2, 33, 600), (1, 130, 513), (3, 50, 900), (16, 5130, 600), (17, 96, 300), (50, 5150, 1300), (61, 130, 5000), (64, 64, 8192), (65, 1, 100), (65, 127, 300), (100, 129, 129),
          (128, 128, 128), (200, 300, 9000), (130, 258, 384), (257, 513, 640), (1001, 999, 200), (512, 384, 1100), (2050, 1030, 600), (3585, 3600, 300), (40, 50, 0), (1, 1, 0)]
KINDS = [(None, True, True), ("relu", True, False), ("gelu", False, True), ("silu", True, True), ("gelu", True, False), (None, False, False)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_dense(env, shape, fmt):
    torch, ssgd = env
    M, N, K = shape
    kinds = KINDS if M * N * K < 1 << 24 else [KINDS[(M + N) % len(KINDS)], KINDS[3]]
    x = _matrix(torch, M, K, M + K).cuda()
    w = (_matrix(torch, N, K, N + K + 1) / math.sqrt(max(K, 1))).cuda()
    a, b = ssgd.mx_quantize(x, fmt), ssgd.mx_quantize(w, "fp4")
    sums, bound = _sums(_host(ssgd.mx_dequantize(a)), _host(ssgd.mx_dequantize(b)), fmt)
    bias, residual = torch.randn(N).cuda(), torch.randn(M, N).cuda()
    for act, with_bias, with_residual in kinds:
        how = dict(bias=bias if with_bias else None, activation=act, residual=residual if with_residual else None)
        out, kept = ssgd.mx_dense(a, b, dtype=torch.float32, keep="same", **how)
        p = sums + (_host(bias) if with_bias else 0)
        wide = bound + U * np.abs(p)
        _within(_host(kept), p, wide)
        y = _act(p, act)
        # slopes are 1.13 at most
        off = 1.13 * wide + _act_error(p, act) + 2 * U * np.abs(y)
        _within(_host(out), y + (_host(residual) if with_residual else 0), off)
        # the other outputs are roundings of these
        half, half_kept = ssgd.mx_dense(a, b, keep="same", **how)
        assert half.dtype == torch.bfloat16 and torch.equal(half, out.to(torch.bfloat16)) and torch.equal(half_kept, kept.to(torch.bfloat16))
        eight, eight_kept = ssgd.mx_dense(a, b, output="fp8", keep="fp8", **how)
        for got, of in ((eight, out), (eight_kept, kept)):
            want = ssgd.mx_quantize(of, "fp8")
            assert got.shape == (M, N) and torch.equal(got.values, want.values) and torch.equal(got.scales, want.scales)
        mixed, mixed_kept = ssgd.mx_dense(a, b, dtype=torch.float32, output="fp8", keep="same", **how)
        assert torch.equal(mixed_kept, kept) and torch.equal(mixed.values, eight.values)
        mixed, mixed_kept = ssgd.mx_dense(a, b, dtype=torch.float32, keep="fp8", **how)
        assert torch.equal(mixed, out) and torch.equal(mixed_kept.values, eight_kept.values) and torch.equal(mixed_kept.scales, eight_kept.scales)
        assert torch.equal(ssgd.mx_dense(a, b, dtype=torch.float32, **how), out)
        # rows quantised on the way: the same bits
        for dtype in (torch.float32, torch.bfloat16):
            z = x.to(dtype)
            q = ssgd.mx_quantize(z, fmt)
            assert torch.equal(ssgd.mx_dense(z, b, format=fmt, **how), ssgd.mx_dense(q, b, dtype=dtype, **how))
            assert torch.equal(ssgd.mx_dense(z, b, format=fmt, output="fp8", **how).values, ssgd.mx_dense(q, b, output="fp8", **how).values)
    # nothing in the epilogue: the product
    assert torch.equal(ssgd.mx_dense(a, b), ssgd.mx_matmul(a, b)) and torch.equal(ssgd.mx_dense(a, b, dtype=torch.float32), ssgd.mx_matmul(a, b, torch.float32))


GATED = [(1, 1, 1), (1, 35, 900), (2, 17, 600), (1, 600, 4100), (3, 50, 900), (16, 2600, 600), (17, 48, 300), (37, 300, 5000), (64, 32, 8192), (65, 1, 100), (65, 63, 300), (100, 65, 129), (128, 64, 128),
         (200, 150, 9000), (130, 129, 384), (257, 257, 640), (1001, 501, 200), (2050, 515, 600), (3585, 1800, 300), (40, 50, 0), (300, 60, 256)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("shape", GATED, ids=str)
def test_gated(env, shape, fmt):
    torch, ssgd = env
    M, H, K = shape
    x = _matrix(torch, M, K, M + K).cuda()
    gate, up = ((_matrix(torch, H, K, H + K + k) / math.sqrt(max(K, 1))).cuda() for k in (1, 2))
    w = ssgd.gate_up(gate, up)
    assert w.shape == (2 * H, K) and torch.equal(w[0::2], gate) and torch.equal(w[1::2], up)
    a, b = ssgd.mx_quantize(x, fmt), ssgd.mx_quantize(w, "fp4")
    p, bound = _sums(_host(ssgd.mx_dequantize(a)), _host(ssgd.mx_dequantize(b)), fmt)
    for act in ("silu", "gelu", "relu", None) if M * H * K < 1 << 23 else ("silu", "gelu"):
        h, kept = ssgd.mx_gated(a, b, act, dtype=torch.float32, keep="same")
        _within(_host(kept), p, bound)
        g, u = p[:, 0::2], p[:, 1::2]
        y = _act(g, act)
        off = (1.13 * bound[:, 0::2] + _act_error(g, act)) * (np.abs(u) + bound[:, 1::2]) + np.abs(y) * bound[:, 1::2] + 2 * U * np.abs(y * u)
        _within(_host(h), y * u, off)
        half, half_kept = ssgd.mx_gated(a, b, act, keep="same")
        assert half.shape == (M, H) and torch.equal(half, h.to(torch.bfloat16)) and torch.equal(half_kept, kept.to(torch.bfloat16))
        eight, eight_kept = ssgd.mx_gated(a, b, act, output="fp8", keep="fp8")
        for got, of in ((eight, h), (eight_kept, kept)):
            want = ssgd.mx_quantize(of, "fp8")
            assert got.shape == of.shape and torch.equal(got.values, want.values) and torch.equal(got.scales, want.scales)
        assert torch.equal(ssgd.mx_gated(a, b, act, output="fp8").values, eight.values) and torch.equal(ssgd.mx_gated(a, b, act, dtype=torch.float32), h)
        mixed, mixed_kept = ssgd.mx_gated(a, b, act, dtype=torch.float32, keep="fp8")
        assert torch.equal(mixed, h) and torch.equal(mixed_kept.values, eight_kept.values)
        for dtype in (torch.float32, torch.bfloat16):
            z = x.to(dtype)
            assert torch.equal(ssgd.mx_gated(z, b, act, format=fmt), ssgd.mx_gated(ssgd.mx_quantize(z, fmt), b, act, dtype=dtype))
    assert torch.equal(ssgd.mx_gated(x, b, format=fmt), ssgd.mx_gated(x, b, "silu", fmt))          # silu unless another is named


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_strides_types_and_alignment(env, rows):
    """Rows, residual and bias at odd places and in other types; a bias and a residual of each type beside an output of the other."""
    torch, ssgd = env
    N, K = 131, 700
    x = _matrix(torch, rows, K, 3).cuda()
    b = ssgd.mx_quantize((_matrix(torch, N, K, 4) / 26).cuda(), "fp4")
    bias, residual = torch.randn(N).to(torch.bfloat16).cuda(), torch.randn(rows, N).to(torch.bfloat16).cuda()
    want = ssgd.mx_dense(x, b, bias=bias.float(), activation="silu", residual=residual.float())
    pad = torch.full((rows, K + 5), float("nan"), device="cuda")
    pad[:, 3:K + 3] = x
    beside = torch.full((rows, N + 3), float("nan"), device="cuda", dtype=torch.bfloat16)
    beside[:, 1:N + 1] = residual
    shifted = torch.full((N + 1,), float("nan"), device="cuda", dtype=torch.bfloat16)
    shifted[1:] = bias
    assert torch.equal(ssgd.mx_dense(pad[:, 3:K + 3], b, bias=shifted[1:], activation="silu", residual=beside[:, 1:N + 1]), want)
    assert torch.equal(ssgd.mx_dense(x, b, bias=bias, activation="silu", residual=residual.float(), dtype=torch.bfloat16), want.to(torch.bfloat16))


@pytest.mark.parametrize("act", [None, "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows", [1, 3, 100])
def test_infinities_nan_and_far_values(env, rows, act):
    """Values of the sums are set through the bias: the activations follow the formulas from the largest to the smallest."""
    torch, ssgd = env
    far = [0.0, -0.0, 1e-38, -1e-30, 1e4, -1e4, 80.0, -80.0, -90.0, -104.0, 300.0, -300.0, 3e38, -3e38, float("inf"), float("nan"), 12.0, -12.0, -6.0, -5.0, 5.0]
    bias = torch.tensor(far).cuda()
    N, K = len(far), 600
    b = ssgd.MxTensor.empty(N, K, "fp4", torch.device("cuda", torch.cuda.current_device()))
    b.values.zero_(), b.scales.zero_()
    out = _host(ssgd.mx_dense(torch.ones(rows, K, device="cuda"), b, bias=bias, activation=act))
    x = np.array(far, dtype=np.float32).astype(float)
    want = _act(x, act)
    for k, v in enumerate(far):
        if math.isnan(v):
            assert np.all(np.isnan(out[:, k]))
        elif math.isinf(v):
            assert np.all(out[:, k] == v)
        else:
            assert np.all(np.abs(out[:, k] - want[k]) <= _act_error(x[k:k + 1], act)[0] + 2.0 ** -126), (v, out[0, k], want[k])
    # a block with a NaN is NaN in 8 bits, what else is in the row is not touched
    q = ssgd.mx_dense(torch.ones(rows, K, device="cuda"), b, bias=bias.repeat(1), activation=act, output="fp8")
    assert torch.all(q.scales[:, 0] == 255) and torch.all(q.values == 0)


def test_blocks_that_are_nan_stay_in_their_row_and_column(env):
    torch, ssgd = env
    M, N, K = 100, 200, 384
    x, w = _matrix(torch, M, K, 1).cuda(), _matrix(torch, N, K, 2).cuda()
    x[7, 5], w[150, 100] = float("inf"), float("nan")
    a, b = ssgd.mx_quantize(x, "fp8"), ssgd.mx_quantize(w, "fp4")
    out = ssgd.mx_dense(a, b, activation="gelu")
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[7], bad[:, 150] = True, True
    assert torch.equal(out.isnan(), bad)
    h, p = ssgd.mx_gated(a, b, output="fp8", keep="fp8")
    assert torch.all(h.scales[7, :4] == 255) and torch.all((h.scales[:, 75 // 32] == 255)) and (p.scales[:, 150 // 32] == 255).all() and int((h.scales[8] == 255).sum()) == 1


def test_refusals_of_the_binding(env):
    torch, ssgd = env
    x, w = torch.randn(4, 200, device="cuda"), ssgd.mx_quantize(torch.randn(6, 200, device="cuda"))
    odd = ssgd.mx_quantize(torch.randn(7, 200, device="cuda"))
    ssgd.mx_dense(x, w)
    for call in (lambda: ssgd.mx_dense(x, w, activation="tanh"), lambda: ssgd.mx_dense(x, w, bias=torch.randn(5, device="cuda")), lambda: ssgd.mx_dense(x, w, bias=torch.randn(6)),
                 lambda: ssgd.mx_dense(x, w, bias=torch.randn(6, device="cuda").double()), lambda: ssgd.mx_dense(x, w, residual=torch.randn(4, 5, device="cuda")),
                 lambda: ssgd.mx_dense(x, w, residual=torch.randn(6, 4, device="cuda").t()), lambda: ssgd.mx_dense(x, w, residual=torch.randn(4, 6)),
                 lambda: ssgd.mx_dense(x, w, output="fp4"), lambda: ssgd.mx_dense(x, w, keep="bf16"), lambda: ssgd.mx_dense(x, w, format="fp6"), lambda: ssgd.mx_dense(x, w, dtype=torch.float16),
                 lambda: ssgd.mx_dense(x[:, :100], w), lambda: ssgd.mx_dense(x, ssgd.mx_quantize(torch.randn(6, 200, device="cuda"), "fp8")), lambda: ssgd.mx_dense(x, x),
                 lambda: ssgd.mx_gated(x, odd), lambda: ssgd.mx_gated(x, w, "swish"), lambda: ssgd.gate_up(x, x[:3]), lambda: ssgd.gate_up(x, x.double())):
        with pytest.raises(ssgd.SsgdError) as e:
            call()
        assert e.value.status == ssgd.EINVAL
    for t in (torch.randn(6, device="cuda", requires_grad=True),):
        with pytest.warns(UserWarning, match="no graph"):
            ssgd.mx_dense(x, w, bias=t)
    for empty in (ssgd.mx_dense(x[:0], w, activation="relu", keep="fp8"), ssgd.mx_gated(x[:0], w, keep="same")):
        assert empty[0].shape[0] == 0 and empty[1].shape == (0, 6)
    assert ssgd.mx_dense(x, ssgd.MxTensor.empty(0, 200, "fp4", x.device), output="fp8").shape == (4, 0)
