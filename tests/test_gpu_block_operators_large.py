"""The operators of a gated feed-forward block where offsets pass 32 bits: the far end against the same operator on a slice of its own."""
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


def _rows(ssgd, q, rows):
    return ssgd.MxTensor(q.values[rows].contiguous(), q.scales[rows].contiguous(), q.format, (len(range(q.shape[0])[rows]), q.shape[1]))


def test_dense_results_of_more_than_2_to_the_32(env):
    torch, ssgd = env
    n, k = 66000, 130
    a, b = ssgd.mx_quantize(torch.randn(n, k, device="cuda")), ssgd.mx_quantize(torch.randn(n, k, device="cuda"))
    bias, residual = torch.randn(n, device="cuda"), torch.empty(n, n, device="cuda", dtype=torch.bfloat16).normal_()
    out, kept = ssgd.mx_dense(a, b, bias=bias, activation="silu", residual=residual, keep="fp8")
    assert out.numel() > 1 << 32 and kept.values.numel() > 1 << 32
    for rows in (slice(0, 256), slice(n - 208, n)):
        # (two steps of 128 columns: the sums are the same in every kernel)
        cols = slice(n - 208, n)
        some, some_kept = ssgd.mx_dense(_rows(ssgd, a, rows), _rows(ssgd, b, cols), bias=bias[cols].contiguous(), activation="silu", residual=residual[rows, cols], keep="fp8")
        assert torch.equal(out[rows, cols], some)
        # blocks of 32 columns from a multiple of 32 on: n - 208 is one of 16
        whole = ssgd.mx_dequantize(_rows(ssgd, kept, rows), torch.float32)[:, n - 192:]
        assert torch.allclose(whole, ssgd.mx_dequantize(some_kept)[:, 16:], rtol=2.0 ** -3, atol=2.0 ** -6 * float(whole.abs().max()))


def test_gated_of_more_than_2_to_the_31(env):
    torch, ssgd = env
    rows, hidden, k, tail = 140000, 16384, 128, 140000 % 256
    a, b = ssgd.mx_quantize(torch.randn(rows, k, device="cuda"), "fp8"), ssgd.mx_quantize(torch.randn(2 * hidden, k, device="cuda") / 11)
    h, p = ssgd.mx_gated(a, b, output="fp8", keep="fp8")
    h2, p2 = ssgd.mx_gated(_rows(ssgd, a, slice(rows - tail, rows)), b, output="fp8", keep="fp8")
    assert p.values.numel() > 1 << 32
    for whole, end in ((h, h2), (p, p2)):
        assert torch.equal(whole.values[-tail:], end.values) and torch.equal(whole.scales[-tail:], end.scales)


def test_gradients_of_more_than_2_to_the_31(env):
    torch, ssgd = env
    rows, hidden = 70000, 16384
    tail = rows % 128                     # the last tile of rows
    dy = torch.empty(rows, hidden, device="cuda", dtype=torch.bfloat16).normal_()
    p = ssgd.MxTensor.empty(rows, 2 * hidden, "fp8", dy.device)
    p.values.random_(0, 120), p.scales.fill_(120)
    d, dt, ht = ssgd.mx_gated_backward(dy, p, "gelu", hidden="fp8")
    d2, dt2, ht2 = ssgd.mx_gated_backward(dy[-tail:], _rows(ssgd, p, slice(rows - tail, rows)), "gelu", hidden="fp8")
    assert d.values.numel() > 1 << 31
    assert torch.equal(d.values[-tail:], d2.values) and torch.equal(d.scales[-tail:], d2.scales)
    for whole, end in ((dt, dt2), (ht, ht2)):
        assert torch.equal(whole.values[:, rows - tail:], end.values) and torch.equal(whole.scales[:, (rows - tail) // 32:], end.scales)
    t = ssgd.mx_transpose(p, "fp4")
    t2 = ssgd.mx_transpose(_rows(ssgd, p, slice(rows - tail, rows)), "fp4")
    assert torch.equal(t.values[:, (rows - tail) // 2:], t2.values) and torch.equal(t.scales[:, (rows - tail) // 32:], t2.scales)
    q, _, _, db = ssgd.mx_dense_backward(dy, None)
    # 70000 normal numbers to a sum, whose root mean square is 265; fp32 sums of 128 of them and fp64 beyond
    want = torch.stack([c.double().sum(0) for c in dy.split(7000)]).sum(0)
    assert torch.allclose(db.double(), want, rtol=0, atol=1e-3) and torch.equal(q.values[-tail:], ssgd.mx_quantize(dy[-tail:], "fp8").values)


def test_norms_of_more_than_2_to_the_31(env):
    torch, ssgd = env
    rows, d, gates, tail = 270000, 8192, 9, 50
    o, s = (torch.empty(rows, d, device="cuda", dtype=torch.bfloat16).normal_() for _ in range(2))
    w, gate = torch.ones(d, device="cuda"), torch.randn(gates, d, device="cuda")
    y, total, rstd_o, rstd = ssgd.block_norm(o, s, w, w, gate=gate, output="fp8")
    end = ssgd.block_norm(o[-tail:], s[-tail:], w, w, gate=gate[-1:], output="fp8")
    assert torch.equal(y.values[-tail:], end[0].values) and all(torch.equal(a[-tail:], b) for a, b in zip((total, rstd_o, rstd), end[1:]))
    do, ds, dpost, dw, dgate = ssgd.block_norm_backward(o, o, total, w, w, rstd_o, rstd, gate=gate, dsum=s)
    do2, ds2, *_ = ssgd.block_norm_backward(o[-tail:], o[-tail:], end[1], w, w, end[2], end[3], gate=gate[-1:], dsum=s[-tail:])
    assert torch.equal(do[-tail:], do2) and torch.equal(ds[-tail:], ds2)
    assert torch.isfinite(dpost).all() and torch.isfinite(dw).all() and torch.isfinite(dgate).all()
    # dw_post is what dgate's sums give with the gates
    assert torch.allclose(dpost, (dgate * gate).sum(0), rtol=1e-4, atol=1e-4 * float(dpost.abs().max()))
