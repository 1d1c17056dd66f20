"""The norms between two blocks with gate and scaled residual, and their gradients, against the formulas in 64 bits, through the public entry points."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _half_place(x, dtype):
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


def _inputs(torch, rows, d, dtype, gates, seed):
    g = torch.Generator().manual_seed(seed)
    one = lambda scale: (torch.randn(rows, d, generator=g) * scale).to(dtype).cuda()  # noqa: E731
    side = lambda *shape: torch.randn(*shape, generator=g).cuda()  # noqa: E731
    gate = None if gates == 0 else 0.5 * side(d) if gates == 1 else 0.5 * side(gates, d)
    return one(3.0), one(1.0), 1 + 0.2 * side(d), 1 + 0.2 * side(d), gate, one(1.0), one(0.5)


def _sum(o, s, post, gate, scale, eps):
    rstd_o = 1 / np.sqrt((o * o).mean(1, keepdims=True) + eps)
    return rstd_o, scale * s + gate * (o * rstd_o * post)


def _check(env, rows, d, dtype, gates, scale, with_dsum=True):
    torch, ssgd = env
    dt = getattr(torch, dtype)
    o, s, post, w, gate, dy, dsum = _inputs(torch, rows, d, dt, gates, rows + d + gates)
    eps = 1e-5
    y, total, rstd_o, rstd = ssgd.block_norm(o, s, post, w, gate=gate, scale=scale, eps=eps)
    assert y.dtype == total.dtype == dt and rstd_o.dtype == rstd.dtype == torch.float32 and rstd.shape == rstd_o.shape == (rows,)
    oh, sh, ph, wh = (_host(x) for x in (o, s, post, w))
    gh = np.ones((1, d)) if gate is None else _host(gate).reshape(-1, d)
    wide = np.repeat(gh, rows // gh.shape[0], 0)
    ro, want = _sum(oh, sh, ph, wide, scale, eps)
    # in 64 bits, then to fp32 and to the type
    assert np.all(np.abs(_host(total) - want) <= (1 + 2.0 ** -14) * _half_place(want, dtype) + U * np.abs(want) * (dtype != "float32") + 1e-40)
    assert np.all(np.abs(_host(rstd_o) - ro[:, 0]) <= 1.01 * U * ro[:, 0])
    t = _host(total)
    r = 1 / np.sqrt((t * t).mean(1, keepdims=True) + eps)
    assert np.all(np.abs(_host(rstd) - r[:, 0]) <= 1.01 * U * r[:, 0])
    # rstd's rounding and two products
    assert np.all(np.abs(_host(y) - t * r * wh) <= 4 * U * np.abs(t * r * wh) + 1.01 * _half_place(t * r * wh, dtype) + 1e-40)
    # 8 bits: the quantisation of the result in fp32
    q, total2, _, _ = ssgd.block_norm(o, s, post, w, gate=gate, scale=scale, eps=eps, output="fp8")
    exact = (total.float() * rstd[:, None]) * w
    want_q = ssgd.mx_quantize(exact, "fp8")
    assert torch.equal(total2, total) and q.shape == (rows, d) and torch.equal(q.values, want_q.values) and torch.equal(q.scales, want_q.scales)

    do, ds, dpost, dw, dgate = ssgd.block_norm_backward(dy, o, total, post, w, rstd_o, rstd, gate=gate, scale=scale, dsum=dsum if with_dsum else None)
    assert do.dtype == ds.dtype == dt and dpost.dtype == dw.dtype == torch.float32 and (dgate is None) == (gate is None)
    dyh, more = _host(dy), _host(dsum) if with_dsum else np.zeros((rows, d))
    mean = lambda x: x.mean(1, keepdims=True)  # noqa: E731
    shat, ohat, gw = t * r, oh * ro, dyh * wh
    G = r * (gw - shat * mean(gw * shat)) + more
    G_size = r * (np.abs(gw) + np.abs(shat) * mean(np.abs(gw * shat))) + np.abs(more)          # of the terms of G
    T = G * wide * ph
    T_size = G_size * np.abs(wide * ph)
    want_o = ro * (T - ohat * mean(T * ohat))
    o_size = ro * (T_size + np.abs(ohat) * mean(T_size * np.abs(ohat)))
    # a thread adds at most sixteen terms in fp32, the rest is fp64 (rows of more than 16384 columns eight at a time); twelve products and sums around them
    off = lambda size: 64 * U * size  # noqa: E731
    assert np.all(np.abs(_host(ds) - scale * G) <= abs(scale) * off(G_size) + 1.01 * _half_place(scale * G, dtype) + 1e-40)
    assert np.all(np.abs(_host(do) - want_o) <= 2 * off(o_size) + 1.01 * _half_place(want_o, dtype) + 1e-40)
    # a unit's at most 64 rows to a thread in fp32, with the products' roundings; fp64 beyond
    sums = (G * ohat, G_size * np.abs(ohat))
    by_gate, size = (x.reshape(gh.shape[0], -1, d).sum(1) for x in sums)
    assert np.all(np.abs(_host(dw) - (dyh * shat).sum(0)) <= 72 * U * np.abs(dyh * shat).sum(0) + 1e-40)
    assert np.all(np.abs(_host(dpost) - (gh * by_gate).sum(0)) <= 140 * U * (np.abs(gh) * size).sum(0) + 1e-40)
    if gate is not None:
        assert dgate.shape == gate.shape and np.all(np.abs(_host(dgate).reshape(-1, d) - ph * by_gate) <= 140 * U * np.abs(ph) * size + 1e-40)


# every form: 64 to 1024 threads a row with eight and sixteen columns each, a row that is read again; one row and more than are at work at a time
SHAPES = [(1, 1, 0), (1, 3001, 1), (3, 7, 1), (4, 64, 2), (2, 511, 0), (9, 512, 3), (7, 513, 7), (4, 1024, 1), (3, 1025, 0), (6, 2048, 2), (2, 2049, 1), (3, 4096, 3), (2, 4097, 1), (3, 8192, 0),
          (2, 8193, 2), (2, 16384, 1), (3, 16385, 3), (2, 20000, 1), (5000, 40, 1), (3000, 1030, 50), (1100, 5000, 1), (600, 9000, 4), (300, 16400, 2), (2000, 100, 2000), (20000, 24, 1), (1000, 600, 8)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_gradients(env, shape, dtype):
    _check(env, *shape[:2], dtype, shape[2], 0.75)


@pytest.mark.parametrize("scale", [1.0, 0.0, -2.5])
def test_scales_of_the_residual(env, scale):
    _check(env, 30, 300, "float32", 3, scale, with_dsum=False)


def test_gradients_against_differences(env):
    torch, ssgd = env
    rows, d, eps, scale = 4, 70, 1e-5, 0.6
    o, s, post, w, gate, dy, dsum = _inputs(torch, rows, d, torch.float32, 2, 5)
    x = {"o": _host(o), "s": _host(s), "post": _host(post), "w": _host(w), "gate": _host(gate)}
    dyh, dsh = _host(dy), _host(dsum)

    def objective(v):
        _, t = _sum(v["o"], v["s"], v["post"], np.repeat(v["gate"], 2, 0), scale, eps)
        return float((dyh * (t / np.sqrt((t * t).mean(1, keepdims=True) + eps) * v["w"]) + dsh * t).sum())
    _, total, rstd_o, rstd = ssgd.block_norm(o, s, post, w, gate=gate, scale=scale, eps=eps)
    got = dict(zip(("o", "s", "post", "w", "gate"), ssgd.block_norm_backward(dy, o, total, post, w, rstd_o, rstd, gate=gate, scale=scale, dsum=dsum)))
    h = 1e-5
    for name, places in (("o", ((0, 0), (3, 69))), ("s", ((1, 33), (2, 5))), ("post", ((0,), (69,))), ("w", ((35,), (1,))), ("gate", ((0, 3), (1, 60)))):
        for at in places:
            up, down = ({**x, name: x[name].copy()} for _ in range(2))
            up[name][at] += h
            down[name][at] -= h
            assert abs((objective(up) - objective(down)) / (2 * h) - float(got[name][at])) < 2e-5


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("d", [100, 1000, 3000, 6000, 10000, 17000])
def test_strides_alignment_and_side_types_do_not_change_results(env, d, dtype):
    torch, ssgd = env
    dt = getattr(torch, dtype)
    rows = 6
    o, s, post, w, gate, dy, dsum = _inputs(torch, rows, d, dt, 3, d)
    post, w, gate = (x.to(torch.bfloat16) for x in (post, w, gate))
    want = ssgd.block_norm(o, s, post.float(), w.float(), gate=gate.float(), scale=0.9)
    want_back = ssgd.block_norm_backward(dy, o, want[1], post.float(), w.float(), want[2], want[3], gate=gate.float(), scale=0.9, dsum=dsum)

    def inside(x, left):
        wide = torch.full((x.shape[0], d + 9), float("nan"), device="cuda", dtype=x.dtype)
        wide[:, left:left + d] = x
        return wide[:, left:left + d]
    got = ssgd.block_norm(inside(o, 1), inside(s, 3), post, w, gate=inside(gate, 5), scale=0.9)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    back = ssgd.block_norm_backward(inside(dy, 7), inside(o, 2), inside(want[1], 1), post, w, want[2], want[3], gate=inside(gate, 5), scale=0.9, dsum=inside(dsum, 3))
    assert all(torch.equal(a, b) for a, b in zip(back, want_back))


@pytest.mark.parametrize("d", [300, 5000, 17000])
def test_rows_that_fp32_squares_do_not_hold(env, d):
    torch, ssgd = env
    g = torch.Generator().manual_seed(d)
    o = torch.randn(3, d, generator=g).cuda() * torch.tensor([1e30, 1e-30, 1.0]).cuda()[:, None]
    s = torch.randn(3, d, generator=g).cuda() * torch.tensor([1.0, 1.0, 1e25]).cuda()[:, None]
    one = torch.ones(d, device="cuda")
    y, total, rstd_o, rstd = ssgd.block_norm(o, s, one, one, eps=0.0)
    ro, want = _sum(_host(o), _host(s), 1.0, 1.0, 1.0, 0.0)
    assert np.all(np.abs(_host(rstd_o) / ro[:, 0] - 1) <= 1.01 * U) and np.all(np.abs(_host(total) - want) <= 1.01 * U * np.abs(want))
    t = _host(total)
    assert np.all(np.abs(_host(rstd) * np.sqrt((t * t).mean(1)) - 1) <= 1.01 * U) and np.all(np.isfinite(_host(y)))


def test_infinities_and_nan_stay_in_their_row(env):
    torch, ssgd = env
    o, s, post, w, gate, dy, dsum = _inputs(torch, 8, 200, torch.bfloat16, 2, 3)
    o[2, 5], s[5, 7] = float("nan"), float("inf")
    y, total, rstd_o, rstd = ssgd.block_norm(o, s, post, w, gate=gate)
    bad = torch.zeros(8, dtype=torch.bool, device="cuda")
    bad[2] = True
    assert torch.equal(total.isnan().any(1), bad) and torch.isinf(total[5, 7])
    bad[5] = True
    assert torch.equal(y.isnan().any(1), bad)
    do, ds, *_ = ssgd.block_norm_backward(dy, o, total, post, w, rstd_o, rstd, gate=gate, dsum=dsum)
    assert torch.isfinite(do[~bad]).all() and torch.isfinite(ds[~bad]).all()


def test_refusals_of_the_binding(env):
    torch, ssgd = env
    o, s, post, w, gate, dy, dsum = _inputs(torch, 6, 40, torch.float32, 3, 1)
    y, total, rstd_o, rstd = ssgd.block_norm(o, s, post, w, gate=gate)
    for call in (lambda: ssgd.block_norm(o, s[:5], post, w), lambda: ssgd.block_norm(o, s.to(torch.bfloat16), post, w), lambda: ssgd.block_norm(o, s, post[:39], w), lambda: ssgd.block_norm(o, s, post, w.cpu()),
                 lambda: ssgd.block_norm(o, s, post, w, gate=torch.ones(4, 40, device="cuda")), lambda: ssgd.block_norm(o, s, post, w, gate=torch.ones(3, 39, device="cuda")),
                 lambda: ssgd.block_norm(o, s, post, w, gate=torch.ones(40)), lambda: ssgd.block_norm(o, s, post, w, gate=torch.ones(0, 40, device="cuda")), lambda: ssgd.block_norm(o, s, post, w, output="fp4"),
                 lambda: ssgd.block_norm(o, s, post, w, eps=-1.0), lambda: ssgd.block_norm(o, s, post, w, scale=float("nan")), lambda: ssgd.block_norm(o, s, post, w, scale=1e39),
                 lambda: ssgd.block_norm(o, s, post, w, gate=gate.double()), lambda: ssgd.block_norm(o.cpu(), s, post, w),
                 lambda: ssgd.block_norm_backward(dy, o, total, post, w, rstd_o[:5], rstd), lambda: ssgd.block_norm_backward(dy, o, total, post, w, rstd_o, rstd.double()),
                 lambda: ssgd.block_norm_backward(dy, o, total[:, :39], post, w, rstd_o, rstd), lambda: ssgd.block_norm_backward(dy, o, total, post, w, rstd_o, rstd, dsum=dsum.to(torch.bfloat16))):
        with pytest.raises(ssgd.SsgdError) as e:
            call()
        assert e.value.status == ssgd.EINVAL
    with pytest.warns(UserWarning, match="no graph"):
        ssgd.block_norm(o, s, post, w, gate=gate.clone().requires_grad_())
    y, total, rstd_o, rstd = ssgd.block_norm(o[:0], s[:0], post, w, output="fp8")
    assert y.shape == (0, 40) and total.shape == (0, 40) and rstd.shape == (0,)
    do, ds, dpost, dw, dgate = ssgd.block_norm_backward(dy[:0], o[:0], total, post, w, rstd_o, rstd, gate=gate)
    assert do.shape == (0, 40) and float(dpost.abs().sum() + dw.abs().sum() + dgate.abs().sum()) == 0.0
