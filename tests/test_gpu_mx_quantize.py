"""Microscaled quantisation against the formats' tables, bit for bit, through the public entry points."""
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


def _check(q, x, fmt):
    """Codes and scales of an MxTensor against those of the matrix x (64 bits)."""
    codes, scales = ref.quantize(x, fmt)
    assert q.shape == x.shape and q.format == fmt
    got = ref.unpack(q.values.cpu().numpy(), fmt)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    bit = 8 if fmt == "fp4" else 128
    assert np.array_equal(got % bit, codes % bit)
    assert np.array_equal((got >= bit) & (got % bit > 0), (codes >= bit) & (codes % bit > 0))


def _values(torch, rows, cols, dtype, seed):
    """Sizes that differ by columns and rows, ties of both formats, zeros, blocks of zeros."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    ties = torch.randint(-64, 65, (rows, cols), generator=g) / 8.0
    x = torch.where(torch.rand(rows, cols, generator=g) < 0.3, ties, x)
    x = torch.where(torch.rand(rows, cols, generator=g) < 0.1, torch.zeros(()), x)
    if cols > 40:
        x[:, 32:64] = 0
    return x.to(dtype)


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (3, 127), (2, 128), (5, 129), (33, 64), (127, 255), (128, 128), (129, 300), (1, 3072), (257, 1000)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rows_columns_and_both(env, shape, dtype, fmt):
    torch, ssgd = env
    x = _values(torch, *shape, getattr(torch, dtype), shape[0] + shape[1])
    d, h = x.cuda(), _host(x)
    other = "fp8" if fmt == "fp4" else "fp4"
    _check(ssgd.mx_quantize(d, fmt), h, fmt)
    _check(ssgd.mx_quantize_transposed(d, fmt), h.T, fmt)
    for f, t in ((fmt, other), (fmt, fmt)):
        a, b = ssgd.mx_quantize_both(d, f, t)
        _check(a, h, f)
        _check(b, h.T, t)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_misaligned_matrices(env, dtype, fmt):
    torch, ssgd = env
    room = _values(torch, 70, 301, getattr(torch, dtype), 9).cuda()
    for view in (room[:, 1:200], room[:, 8:264], room[3::7], room[1:2, 5:], room[:0], room[:, :0], room[:, 300:]):
        a, b = ssgd.mx_quantize_both(view, fmt, fmt)
        _check(ssgd.mx_quantize(view, fmt), _host(view), fmt)
        _check(a, _host(view), fmt)
        if view.numel():
            _check(b, _host(view).T, fmt)
        back = ssgd.mx_dequantize(a)
        assert back.shape == view.shape and np.array_equal(_host(back), ref.rounded(_host(view), fmt))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_row_end(env, dtype):
    """Whatever lies around a matrix, and wherever in a thread's eight columns its rows end, the result is that of the matrix alone."""
    torch, ssgd = env
    for cols in [*range(1, 42), *range(120, 138), 520, 643]:
        x = _values(torch, 37, cols, getattr(torch, dtype), cols).cuda()
        room = torch.full((39, cols + 9), float("nan"), dtype=x.dtype, device="cuda")
        room[1:38, 3:3 + cols] = x
        inside = room[1:38, 3:3 + cols]
        for f in ("fp4", "fp8"):
            pairs = list(zip(ssgd.mx_quantize_both(x, f, f), ssgd.mx_quantize_both(inside, f, f)))
            pairs.append((pairs[0][0], ssgd.mx_quantize(inside, f)))
            pairs.append((pairs[1][0], ssgd.mx_quantize_transposed(inside, f)))
            assert all(torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales) for a, b in pairs), cols
            assert not torch.any(pairs[0][0].scales == 255), cols


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_the_whole_range_of_fp32(env, fmt):
    """Every exponent, from the numbers below the normal ones to the largest, alone and beside small ones."""
    torch, ssgd = env
    g = torch.Generator().manual_seed(1)
    e = torch.arange(-149, 128).repeat_interleave(2)
    x = torch.ldexp(1 + torch.rand(len(e), 32, generator=g, dtype=torch.float64), e[:, None].double()) * torch.sign(torch.randn(len(e), 32, generator=g))
    x[:, ::3] = torch.ldexp(x[:, ::3], torch.tensor(-7.0))
    x[1::2, 1:] = 0
    x = x.float()
    x[torch.isinf(x)] = 3.4028234663852886e38
    _check(ssgd.mx_quantize(x.cuda(), fmt), _host(x), fmt)
    _check(ssgd.mx_quantize_transposed(x.cuda(), fmt), _host(x).T, fmt)
    q = ssgd.mx_quantize(x.cuda(), fmt)
    assert np.array_equal(_host(ssgd.mx_dequantize(q)).astype(np.float32), ref.rounded(_host(x), fmt).astype(np.float32))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_infinities_and_nan_take_their_block(env, fmt):
    torch, ssgd = env
    x = torch.ones(64, 96)
    x[0, 0], x[1, 40], x[2, 95], x[40, 64] = float("inf"), -float("inf"), float("nan"), float("nan")
    _check(ssgd.mx_quantize(x.cuda(), fmt), _host(x), fmt)
    _check(ssgd.mx_quantize_transposed(x.cuda(), fmt), _host(x).T, fmt)
    for dtype in (torch.float32, torch.bfloat16):
        back = ssgd.mx_dequantize(ssgd.mx_quantize(x.cuda(), fmt), dtype).cpu()
        assert back.dtype == dtype and torch.isnan(back).sum() == 4 * 32
        assert torch.isnan(back[0, :32]).all() and torch.isnan(back[1, 32:64]).all() and torch.isnan(back[2, 64:]).all() and (back[3] == 1).all()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_every_code_reads_back(env, fmt):
    torch, ssgd = env
    codes = np.arange(16 if fmt == "fp4" else 256, dtype=np.uint8)
    codes = codes[codes % 128 != 127] if fmt == "fp8" else codes          # E4M3's NaN, which no quantisation gives
    rows = [0, 1, 100, 127, 200, 246 if fmt == "fp8" else 252]
    q = ssgd.MxTensor.empty(len(rows), 256, fmt, "cuda")
    c = np.resize(codes, (len(rows), 256))
    q.values.copy_(torch.from_numpy(c if fmt == "fp8" else (c[:, 0::2] | (c[:, 1::2] << 4))))
    q.scales.copy_(torch.tensor(rows, dtype=torch.uint8)[:, None].expand(-1, 8))
    want = ref.values_of(c, np.repeat(np.array(rows)[:, None], 8, 1), fmt, 256)
    assert np.array_equal(_host(ssgd.mx_dequantize(q)).astype(np.float32), want.astype(np.float32))
    assert np.array_equal(_host(ssgd.mx_dequantize(q, torch.bfloat16))[2:], want[2:])


def test_another_stream_gives_the_same(env):
    torch, ssgd = env
    x = _values(torch, 300, 500, torch.float32, 3).cuda()
    want = ssgd.mx_quantize_both(x, "fp4", "fp8")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = ssgd.mx_quantize_both(x, "fp4", "fp8")
    s.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales)


def test_refusals(env):
    torch, ssgd = env
    x = torch.zeros(8, 64, device="cuda")
    for bad in (x.cpu(), x.double(), x.half(), x[0], x.t(), x[:, ::2], x.expand(2, 8, 64)):
        for f in (ssgd.mx_quantize, ssgd.mx_quantize_transposed, ssgd.mx_quantize_both):
            with pytest.raises(ssgd.SsgdError) as e:
                f(bad)
            assert e.value.status == ssgd.EINVAL
    for f in (lambda: ssgd.mx_quantize(x, "fp6"), lambda: ssgd.mx_quantize_both(x, "fp4", "int8"), lambda: ssgd.mx_dequantize(x)):
        with pytest.raises(ssgd.SsgdError):
            f()
    q = ssgd.mx_quantize(x)
    with pytest.raises(ssgd.SsgdError):
        ssgd.mx_dequantize(q, torch.float16)
    again = ssgd.MxTensor(q.values, q.scales, q.format, q.shape)
    assert torch.equal(ssgd.mx_dequantize(again), ssgd.mx_dequantize(q))
    for values, scales, f, shape in ((q.values, q.scales[:, :1], "fp4", (8, 64)), (q.values[:, :32], q.scales, "fp4", (8, 64)), (q.values.cpu(), q.scales, "fp4", (8, 64)),
                                     (q.values, q.scales, "fp8", (8, 64)), (q.values, q.scales, "fp4", (8, 200)), (q.values, q.scales, "fp4", (7, 64)),
                                     (q.values, q.scales, "fp6", (8, 64)), (q.values.float(), q.scales, "fp4", (8, 64))):
        with pytest.raises(ssgd.SsgdError):
            ssgd.MxTensor(values, scales, f, shape)


def test_copies_are_matrices_of_their_own(env):
    """A deep copy and a stored matrix keep their values when the first one changes."""
    import copy
    import io
    torch, ssgd = env
    x = torch.randn(9, 200, generator=torch.Generator().manual_seed(3)).cuda()
    for fmt in ("fp4", "fp8"):
        q = ssgd.mx_quantize(x, fmt)
        want = ssgd.mx_dequantize(q)
        stored = io.BytesIO()
        torch.save(q, stored)
        stored.seek(0)
        others = [copy.deepcopy(q), torch.load(stored, weights_only=False)]       # (written a line above)
        q.values.zero_()
        for other in others:
            assert other.shape == (9, 200) and other.format == fmt and torch.equal(ssgd.mx_dequantize(other), want)
        assert not ssgd.mx_dequantize(copy.copy(q)).any()
