"""The root-mean-square norm and its gradients against the formulas in 64 bits, through the public entry points."""
import numpy as np
import pytest

import mx_reference as ref

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24          # half a unit in the last place of fp32, relative


def _half_place(x, dtype):
    """Half the distance of the neighbours of |x| in the type: 24 or 8 binary digits."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 1e-38))) - (24 if dtype == "float32" else 8))


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2003_10579_amd import ssgd
    assert torch.cuda.is_available(), "this test needs the GPU"
    ssgd.lib()
    return torch, ssgd


def _host(x):
    return x.double().cpu().numpy()


def _inputs(torch, rows, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    def one(scale):
        return (torch.randn(rows, d, generator=g) * scale).to(dtype).cuda()
    w = (1 + 0.2 * torch.randn(d, generator=g)).cuda()
    return one(2.0), one(1.0), w, one(1.0), one(0.5)


def _formulas(s, w, eps, dy, dsum):
    rstd = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    xhat = s * rstd
    g = dy * w
    dx = rstd * (g - xhat * (g * xhat).mean(1, keepdims=True)) + dsum
    size = rstd * (np.abs(g) + np.abs(xhat) * np.abs(g * xhat).mean(1, keepdims=True)) + np.abs(dsum)      # of the terms of dx
    return rstd[:, 0], xhat * w, dx, (dy * xhat).sum(0), size, np.abs(dy * xhat).sum(0)


# every form: 64, 256 and 1024 threads a row with eight and sixteen columns each, a row that is read twice; more rows than are at work at a time
SHAPES = [(1, 1), (1, 3072), (3, 7), (5, 64), (2, 511), (9, 512), (7, 513), (4, 1024), (3, 1025), (6, 2048), (2, 2049), (3, 4096), (2, 4097), (3, 8192),
          (2, 8193), (2, 16384), (3, 16385), (2, 20000), (5000, 40), (3000, 1030), (1100, 5000), (600, 16400)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_gradients(env, shape, dtype):
    torch, ssgd = env
    rows, d = shape
    dt = getattr(torch, dtype)
    x, r, w, dy, dsum = _inputs(torch, rows, d, dt, rows + d)
    total = (x.float() + r.float()).to(dt)
    y, s, rstd = ssgd.rmsnorm(x, w, residual=r, eps=1e-5)
    assert torch.equal(s, total) and y.dtype == dt and rstd.dtype == torch.float32
    rs, yw, dxw, dww, size, dwsize = _formulas(_host(total), _host(w), 1e-5, _host(dy), _host(dsum))
    # a thread adds at most 16 squares (or 8 at a time) in fp32, the rest is fp64; then the root and a quotient
    assert np.all(np.abs(_host(rstd) - rs) <= 16 * U32 * rs)
    assert np.all(np.abs(_host(y) - yw) <= 20 * U32 * np.abs(yw) + 1.01 * _half_place(yw, dtype) + 1e-40)
    dx, dw = ssgd.rmsnorm_backward(dy, s, w, rstd, dsum=dsum)
    assert dx.dtype == dt and dw.dtype == torch.float32
    assert np.all(np.abs(_host(dx) - dxw) <= 64 * U32 * size + 1.01 * _half_place(dxw, dtype) + 1e-40)
    # a thread adds the rows that it takes, at most 16 of 8192 or one in 512, in fp32
    assert np.all(np.abs(_host(dw) - dww) <= (24 + rows / 512) * U32 * dwsize + 1e-40)
    # without a residual, and without a gradient past the norm
    y2, s2, rstd2 = ssgd.rmsnorm(total, w, eps=1e-5)
    assert s2 is total and torch.equal(y, y2) and torch.equal(rstd, rstd2)
    dx2, dw2 = ssgd.rmsnorm_backward(dy, s, w, rstd)
    dxw2 = dxw - _host(dsum)
    assert np.all(np.abs(_host(dx2) - dxw2) <= 64 * U32 * size + 1.01 * _half_place(dxw2, dtype) + 1e-40) and torch.equal(dw, dw2)
    # the same in 8 bits: the scale byte and values are those of y, but where fp32 leaves y on one side or the other of a threshold
    q, s3, _ = ssgd.rmsnorm(x, w, residual=r, eps=1e-5, output="fp8")
    assert torch.equal(s3, s) and q.shape == (rows, d) and q.format == "fp8"
    codes, scales = ref.quantize(yw, "fp8")
    got, got_scales = q.values.cpu().numpy(), q.scales.cpu().numpy()
    assert got.shape == codes.shape and got_scales.shape == scales.shape
    other = got_scales != scales
    assert other.mean() <= 1e-3 if other.size > 5000 else other.sum() <= 1
    same = ~np.repeat(other, 32, 1)
    off = same & (got % 128 != codes % 128)
    assert off.sum() <= 1 + 1e-4 * off.size
    assert np.all(np.abs(got[off].astype(int) % 128 - codes[off].astype(int) % 128) <= 1)
    assert np.all(got[:, d:] == 0) and np.all(got_scales[:, -(-d // 32):] == 0)


def test_gradients_against_differences(env):
    """Central differences of the whole forward pass in 64 bits against the backward kernel."""
    torch, ssgd = env
    rows, d = 3, 70
    x, r, w, dy, dsum = _inputs(torch, rows, d, torch.float32, 5)
    s, wh, dyh, dsh = _host(x + r), _host(w), _host(dy), _host(dsum)

    def objective(s, w):
        return float((dyh * (s / np.sqrt((s * s).mean(1, keepdims=True) + 1e-5) * w) + dsh * s).sum())
    _, total, rstd = ssgd.rmsnorm(x, w, residual=r, eps=1e-5)
    dx, dw = ssgd.rmsnorm_backward(dy, total, w, rstd, dsum=dsum)
    h = 1e-5
    for i, j in ((0, 0), (1, 33), (2, 69)):
        e = np.zeros_like(s); e[i, j] = h
        assert abs((objective(s + e, wh) - objective(s - e, wh)) / (2 * h) - float(dx[i, j])) < 1e-5
    for j in (0, 35, 69):
        e = np.zeros_like(wh); e[j] = h
        assert abs((objective(s, wh + e) - objective(s, wh - e)) / (2 * h) - float(dw[j])) < 1e-5


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("d", [100, 1000, 3000, 6000, 17000])
def test_strides_alignment_and_a_weight_in_bf16_do_not_change_results(env, d, dtype):
    torch, ssgd = env
    dt = getattr(torch, dtype)
    x, r, w, dy, dsum = _inputs(torch, 9, d, dt, d)
    w = w.to(torch.bfloat16)
    want = ssgd.rmsnorm(x, w.float(), residual=r)
    want_dx, want_dw = ssgd.rmsnorm_backward(dy, want[1], w.float(), want[2], dsum=dsum)
    def strided(t, pad, offset):
        room = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
        room[:, offset:offset + t.shape[1]] = t
        return room[:, offset:offset + t.shape[1]]
    for pad, offset in ((8, 8), (3, 1), (16, 5)):
        v = [strided(t, pad, offset) for t in (x, r, dy, dsum)]
        got = ssgd.rmsnorm(v[0], w, residual=v[1])
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        dx, dw = ssgd.rmsnorm_backward(v[2], strided(got[1], pad, offset), w, got[2], dsum=v[3])
        assert torch.equal(dx, want_dx) and torch.equal(dw, want_dw)


def test_empty_zero_and_infinite_rows(env):
    torch, ssgd = env
    w = torch.ones(96, device="cuda")
    x = torch.zeros(0, 96, device="cuda")
    y, s, rstd = ssgd.rmsnorm(x, w, residual=x)
    assert y.shape == (0, 96) and rstd.shape == (0,)
    dx, dw = ssgd.rmsnorm_backward(y, s, w, rstd)
    assert dx.shape == (0, 96) and torch.equal(dw, torch.zeros(96, device="cuda"))
    x = torch.zeros(4, 96, device="cuda")
    x[1, 5], x[2, 5], x[3] = float("nan"), float("inf"), 1e-30
    for out in (None, "fp8"):
        y, s, rstd = ssgd.rmsnorm(x, w, output=out)
        y = y if out is None else ssgd.mx_dequantize(y)
        assert torch.all(y[0] == 0) and torch.isnan(y[1]).all() and float(rstd[0]) == pytest.approx(1000.0, rel=1e-6)
        assert torch.isnan(y[2, 5]) and float(rstd[2]) == 0 and torch.isfinite(y[3]).all()
    y, s, rstd = ssgd.rmsnorm(torch.zeros(1, 8, device="cuda"), w[:8], eps=0.0)
    assert torch.isnan(y).all() and torch.isinf(rstd).all()         # 0 / 0, as the formula has it


def test_nothing_is_written_beside_the_outputs(env):
    """Through the C entry, with room around every output."""
    torch, ssgd = env
    L = ssgd.lib()
    for rows, d in ((3, 100), (2, 1500), (2, 5000), (2, 17000)):
        x = torch.randn(rows, d, device="cuda")
        w = torch.ones(d, device="cuda")
        room = lambda n: torch.full((n + 64,), 7.0, device="cuda")  # noqa: E731
        total, y, rstd, dx, dw = room(rows * d), room(rows * d), room(rows), room(rows * d), room(d)
        at = lambda t: t.data_ptr() + 128  # noqa: E731
        stream = torch.cuda.current_stream().cuda_stream
        assert L.ssgd_rmsnorm(x.data_ptr(), d, x.data_ptr(), d, w.data_ptr(), 0, 0, rows, d, 1e-6, at(total), d, at(y), d, None, None, at(rstd), stream) == 0
        floats = L.ssgd_rmsnorm_work_floats(rows, d)
        work = room(floats)
        assert L.ssgd_rmsnorm_backward(x.data_ptr(), d, at(total), d, w.data_ptr(), 0, 0, at(rstd), None, 0, rows, d, at(dx), d, at(dw), at(work), stream) == 0
        torch.cuda.synchronize()
        for t, n in ((total, rows * d), (y, rows * d), (rstd, rows), (dx, rows * d), (dw, d), (work, floats)):
            assert torch.all(t[:32] == 7) and torch.all(t[32 + n:] == 7) and not torch.any(t[32:32 + n] == 7)
        # in place: the sum over the residual, the gradient over the one that came in
        r = x.clone()
        assert L.ssgd_rmsnorm(x.data_ptr(), d, r.data_ptr(), d, w.data_ptr(), 0, 0, rows, d, 1e-6, r.data_ptr(), d, at(y), d, None, None, at(rstd), stream) == 0
        assert torch.equal(r, x + x)
        g = x.clone()
        assert L.ssgd_rmsnorm_backward(g.data_ptr(), d, r.data_ptr(), d, w.data_ptr(), 0, 0, at(rstd), None, 0, rows, d, g.data_ptr(), d, None, None, stream) == 0
        assert torch.equal(g.reshape(-1), dx[32:32 + rows * d])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_row_end(env, dtype):
    """Whatever lies around the rows, and wherever in a thread's eight columns they end, the results are those of the rows alone."""
    torch, ssgd = env
    for d in [*range(1, 42), *range(504, 522), 1030, 1537, 4103, 8197]:
        x, r, w, dy, dsum = _inputs(torch, 3, d, getattr(torch, dtype), d)
        y, s, rstd = ssgd.rmsnorm(x, w, residual=r)
        want = (y, s, rstd) + ssgd.rmsnorm_backward(dy, s, w, rstd, dsum=dsum)
        def within(t):
            room = torch.full((5, d + 9), float("nan"), dtype=t.dtype, device="cuda")
            room[1:4, 3:3 + d] = t
            return room[1:4, 3:3 + d]
        y2, s2, rstd2 = ssgd.rmsnorm(within(x), w, residual=within(r))
        got = (y2, s2, rstd2) + ssgd.rmsnorm_backward(within(dy), within(s2), w, rstd2, dsum=within(dsum))
        assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(want, got)), d
        q, q2 = ssgd.rmsnorm(x, w, residual=r, output="fp8")[0], ssgd.rmsnorm(within(x), w, residual=within(r), output="fp8")[0]
        assert torch.equal(q.values, q2.values) and torch.equal(q.scales, q2.scales), d


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("d", [7, 50, 513, 1000, 1537, 2055, 4000, 6001, 8200, 17001])
def test_in_place(env, d, dtype):
    """The sum over x or over the residual, the gradient over dy or over dsum: as into arrays of their own."""
    torch, ssgd = env
    L, dt, kind, rows = ssgd.lib(), getattr(torch, dtype), 0 if dtype == "float32" else 1, 2500 if d < 5000 else 700
    x, r, w, dy, dsum = _inputs(torch, rows, d, dt, d)
    y, s, rstd = ssgd.rmsnorm(x, w, residual=r)
    dx, _ = ssgd.rmsnorm_backward(dy, s, w, rstd, dsum=dsum)
    stream = torch.cuda.current_stream().cuda_stream
    for over_x in (True, False):
        a, b, y2, rstd2 = x.clone(), r.clone(), torch.empty_like(x), torch.empty_like(rstd)
        to = a if over_x else b
        assert L.ssgd_rmsnorm(a.data_ptr(), d, b.data_ptr(), d, w.data_ptr(), kind, 0, rows, d, 1e-6, to.data_ptr(), d, y2.data_ptr(), d, None, None,
                              rstd2.data_ptr(), stream) == 0
        assert torch.equal(to, s) and torch.equal(y2, y) and torch.equal(rstd2, rstd)
        a, b = dy.clone(), dsum.clone()
        to = a if over_x else b
        assert L.ssgd_rmsnorm_backward(a.data_ptr(), d, s.data_ptr(), d, w.data_ptr(), kind, 0, rstd.data_ptr(), b.data_ptr(), d, rows, d, to.data_ptr(), d,
                                       None, None, stream) == 0
        assert torch.equal(to, dx)


def test_another_stream_gives_the_same(env):
    torch, ssgd = env
    x, r, w, dy, dsum = _inputs(torch, 700, 3000, torch.bfloat16, 1)
    y, s, rstd = ssgd.rmsnorm(x, w, residual=r)
    want = (y, s, rstd) + ssgd.rmsnorm_backward(dy, s, w, rstd, dsum=dsum)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y, s, rstd = ssgd.rmsnorm(x, w, residual=r)
        got = (y, s, rstd) + ssgd.rmsnorm_backward(dy, s, w, rstd, dsum=dsum)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals(env):
    torch, ssgd = env
    x = torch.zeros(4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    rstd = torch.ones(4, device="cuda")
    for call in (lambda: ssgd.rmsnorm(x.cpu(), w), lambda: ssgd.rmsnorm(x.half(), w), lambda: ssgd.rmsnorm(x[0], w), lambda: ssgd.rmsnorm(x.t(), w),
                 lambda: ssgd.rmsnorm(x, w[:5]), lambda: ssgd.rmsnorm(x, w.half()), lambda: ssgd.rmsnorm(x, w.cpu()), lambda: ssgd.rmsnorm(x, w, residual=x[:2]),
                 lambda: ssgd.rmsnorm(x, w, residual=x.bfloat16()), lambda: ssgd.rmsnorm(x, w, eps=-1.0), lambda: ssgd.rmsnorm(x, w, eps=float("nan")),
                 lambda: ssgd.rmsnorm(x, w, output="fp4"), lambda: ssgd.rmsnorm(x[:, :0], w[:0]), lambda: ssgd.rmsnorm_backward(x, x[:, :5], w, rstd),
                 lambda: ssgd.rmsnorm_backward(x, x, w, rstd[:2]), lambda: ssgd.rmsnorm_backward(x, x, w, rstd, dsum=x.bfloat16()),
                 lambda: ssgd.rmsnorm_backward(x, x.bfloat16(), w, rstd), lambda: ssgd.rmsnorm_backward(x[:, :0], x[:, :0], w[:0], rstd)):
        with pytest.raises(ssgd.SsgdError) as e:
            call()
        assert e.value.status == ssgd.EINVAL


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("d", [5, 400, 900, 1900, 4000, 8000, 16000, 17000])
def test_rows_whose_squares_fp32_does_not_hold(env, d, dtype, residual):
    """Rows from 1e-30 to 3e37 beside ordinary ones, eps from nothing to past fp32: s^2 leaves fp32 on both sides, rstd and y do not."""
    torch, ssgd = env
    dt = getattr(torch, dtype)
    levels = torch.tensor([1.0, 1e25, 1e-25, 3e19, 1e-30, 3e37, 2.0, 1e20, 1e-20, 0.0])[:, None].cuda()
    g = torch.Generator().manual_seed(d)
    x = ((0.5 + torch.rand(10, d, generator=g)) * torch.randn(10, d, generator=g).sign()).cuda()
    r = (x * 0.5 * levels).to(dt) if residual else None
    x = (x * levels).to(dt)
    w = (1 + 0.2 * torch.randn(d, generator=g)).cuda()
    dy = torch.randn(10, d, generator=g).to(dt).cuda()
    total = x if r is None else (x.float() + r.float()).to(dt)
    for eps in (1e-6, 1e-50, 1e39):
        y, s, rstd = ssgd.rmsnorm(x, w, residual=r, eps=eps)
        assert torch.equal(s, total)
        h = _host(total)
        rs = 1 / np.sqrt((h * h).mean(1) + eps)
        # 16 terms at most in fp32, a root and a quotient; below the normal numbers 2^-149 is a place
        assert np.all(np.abs(_host(rstd) - rs) <= 16 * U32 * rs + 2.0 ** -149)
        yw = h * rs[:, None] * _host(w)
        assert np.all(np.abs(_host(y) - yw) <= 20 * U32 * np.abs(yw) + 1.01 * _half_place(yw, dtype) + np.abs(h * _host(w)) * 2.0 ** -149 + 1e-40)
        q = ssgd.rmsnorm(x, w, residual=r, eps=eps, output="fp8")[0]
        back = _host(ssgd.mx_dequantize(q))
        # half a place of E4M3 at most 2^-4 of a value, and 2^-10 times the scale, 2^-8 of the block's largest value, below its normal numbers; a
        # block's largest value may be cut off at 448 / 512
        block = np.abs(np.pad(yw, ((0, 0), (0, -d % 32)))).reshape(10, -1, 32).max(2).repeat(32, 1)[:, :d]
        assert np.all(np.abs(back - yw) <= (0.125 + 2.0 ** -10) * np.abs(yw) + 2.0 ** -17 * block + np.abs(h * _host(w)) * 2.0 ** -148 + 1e-38)
        if eps == 1e-6:
            dx, dw = ssgd.rmsnorm_backward(dy, s, w, rstd)
            _, _, dxw, dww, size, dwsize = _formulas(h, _host(w), eps, _host(dy), 0.0)
            assert np.all(np.abs(_host(dx) - dxw) <= 64 * U32 * size + 1.01 * _half_place(dxw, dtype) + 1e-38)
            assert np.all(np.abs(_host(dw) - dww) <= 24 * U32 * dwsize + np.abs(_host(dy) * h).sum(0) * 2.0 ** -149 + 1e-40)


@pytest.mark.parametrize("dtype,d,teams", [("float32", 20, 4096), ("bfloat16", 20, 4096), ("bfloat16", 600, 3072), ("bfloat16", 1030, 1024), ("bfloat16", 2100, 768),
                                           ("float32", 4200, 256), ("bfloat16", 4200, 256), ("bfloat16", 9000, 256), ("bfloat16", 17000, 256)])
def test_gradient_of_the_weight_over_very_many_rows(env, dtype, d, teams):
    """1200 rows to each team of threads, equal ones, whose products add up in one direction: however many, at most 64 of them are added in fp32 before
    they join a wider sum."""
    torch, ssgd = env
    dt, rows = getattr(torch, dtype), teams * 1200 + 37
    g = torch.Generator().manual_seed(d)
    dy, s = ((0.1 + torch.rand(1, d, generator=g)).to(dt).cuda() for _ in range(2))
    rstd = torch.full((rows,), 0.9, device="cuda")
    want = rows * _host(dy)[0] * _host(s)[0] * float(rstd[0])
    _, dw = ssgd.rmsnorm_backward(dy.expand(rows, d).contiguous(), s.expand(rows, d).contiguous(), torch.ones(d, device="cuda"), rstd)
    # two products, 64 sums, the rounding of a team's sum, those of four teams and the result's
    assert np.all(np.abs(_host(dw) - want) <= 72 * U32 * want)


def test_nothing_is_written_beside_the_work_area_of_many_long_rows(env):
    torch, ssgd = env
    L, rows, d = ssgd.lib(), 16500, 16390
    dy, w, rstd = torch.ones(rows, d, device="cuda", dtype=torch.bfloat16), torch.ones(d, device="cuda"), torch.ones(rows, device="cuda")
    floats = L.ssgd_rmsnorm_work_floats(rows, d)
    work, dw, dx = torch.full((floats + 64,), 7.0, device="cuda"), torch.full((d + 64,), 7.0, device="cuda"), torch.empty_like(dy)
    assert L.ssgd_rmsnorm_backward(dy.data_ptr(), d, dy.data_ptr(), d, w.data_ptr(), 1, 0, rstd.data_ptr(), None, 0, rows, d, dx.data_ptr(), d, dw.data_ptr() + 128,
                                   work.data_ptr() + 128, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.all(dw[32:32 + d] == rows)
    for t, n in ((work, floats), (dw, d)):
        assert torch.all(t[:32] == 7) and torch.all(t[32 + n:] == 7)
