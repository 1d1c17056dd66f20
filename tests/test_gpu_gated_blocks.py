"""The operators of a gated feed-forward block together: trained, captured into a graph, on streams of their own, and one row among others."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2003_10579_amd import lowbit_block, ssgd
    assert torch.cuda.is_available(), "this test needs the GPU"
    ssgd.lib()
    return torch, ssgd, lowbit_block


@pytest.mark.parametrize("state_bits", [8, 32])
def test_gated_blocks_train_reproducibly(env, state_bits):
    torch, _, lowbit_block = env
    runs = [lowbit_block.train_gated(5, rows=333, width=200, hidden=150, blocks=2, state_bits=state_bits, report=None) for _ in range(2)]
    (model, losses), (again, losses2) = runs
    assert np.all(np.isfinite(losses)) and losses == losses2
    assert all(torch.equal(a, b) for a, b in zip(model.up + model.down + model.gate + model.w_in, again.up + again.down + again.gate + again.w_in))


def _reference(torch, model, x, dy):
    """The gradients of sum(out dy) in 64 bits, of the blocks at the values that their quantised weights stand for: nothing else is quantised."""
    from paper_2003_10579_amd import ssgd
    leaf = lambda t: t.detach().double().clone().requires_grad_()  # noqa: E731
    norm = lambda v, w: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    w_in, w_out, gate, bias = ([leaf(t) for t in ts] for ts in (model.w_in, model.w_out, model.gate, model.bias))
    up, down = ([leaf(ssgd.mx_dequantize(q[0])) for q in qs] for qs in (model.q_up, model.q_down))
    x = leaf(x)
    s, y = x, norm(x, w_in[0])
    for k in range(model.blocks):
        p = y @ up[k].t()
        h = torch.nn.functional.silu(p[:, 0::2]) * p[:, 1::2]
        s = s + gate[k] * norm(h @ down[k].t() + bias[k], w_out[k])
        y = norm(s, w_in[k + 1])
    y.backward(dy.double())
    return y.detach(), x.grad, [t.grad for t in w_in + w_out + gate + bias + up + down]


def test_gradients_of_the_blocks(env):
    """Against autograd in 64 bits.  Activations and gradients are in 8 bits (a rounding is off by 2^-4 at most, 2^-5.4 as a mean square over a binade's steps), right operands of the
    weights' products in 4 (2^-2 at most, under 2^-3 as a mean square) and the transposed weights are quantised along the other direction (another 2^-3): with at most two
    blocks these errors, independent of each other, add up to less than 0.35 of a gradient's norm."""
    torch, ssgd, lowbit_block = env
    model = lowbit_block.GatedBlocks(256, 160, 2, seed=4)
    model.quantize_weights()
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(300, 256, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    out, first, kept = model.forward(x, keep="fp8")
    dx, grads = model.backward(dy, x, first, kept)
    want, want_dx, want_grads = _reference(torch, model, x, dy)
    off = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert off(out, want) < 0.1 and off(dx, want_dx) < 0.35
    for k, (a, b) in enumerate(zip(grads, want_grads)):
        assert a.shape == b.shape and off(a, b) < 0.35, (k, off(a, b))


def test_one_row_among_others(env):
    torch, _, lowbit_block = env
    model = lowbit_block.GatedBlocks(300, 700, 2, seed=2)
    model.quantize_weights()
    x = torch.randn(70, 300, device="cuda").to(torch.bfloat16)
    whole, one = model.answer(x), model.answer(x[3:4])
    # sums in another order: a rounding to bfloat16, or to 8 bits in between, may fall the other way
    assert torch.allclose(one.float(), whole[3:4].float(), rtol=2.0 ** -5, atol=2.0 ** -5 * float(whole.float().abs().max()))
    assert torch.equal(model.answer(x), whole)


def test_captured_and_replayed(env):
    """Forward and backward pass in one graph, replayed with new inputs, with eager work between the replays; and two graphs at once."""
    torch, _, lowbit_block = env
    model = lowbit_block.GatedBlocks(256, 200, 2, seed=3)
    model.quantize_weights()
    def all_of(x, dy):
        out, first, kept = model.forward(x, keep="fp8")
        dx, grads = model.backward(dy, x, first, kept)
        return [out, dx] + grads
    xs = [torch.randn(130, 256, device="cuda").to(torch.bfloat16) for _ in range(2)]
    dys = [torch.randn(130, 256, device="cuda").to(torch.bfloat16) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(2):
            all_of(xs[k], dys[k])
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(all_of(xs[k], dys[k]))
        graphs.append(graph)
    for turn in range(3):
        for k in range(2):
            xs[k].copy_(torch.randn(130, 256, device="cuda")), dys[k].copy_(torch.randn(130, 256, device="cuda"))
        want = [all_of(xs[k], dys[k]) for k in range(2)]
        torch.cuda.synchronize()
        for k in ((0, 1), (1, 0), (0, 1))[turn]:
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k]))


def test_two_streams_at_once(env):
    torch, _, lowbit_block = env
    model = lowbit_block.GatedBlocks(512, 300, 1, seed=5)
    model.quantize_weights()
    x = torch.randn(500, 512, device="cuda").to(torch.bfloat16)
    want = [model.answer(x[:n]) for n in (500, 20, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [None] * 3
    for _ in range(5):
        for k, n in enumerate((500, 20, 1)):
            with torch.cuda.stream(streams[k]):
                got[k] = model.answer(x[:n])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows", [1, 2, 12, 40, 70])
def test_answers_captured_and_replayed(env, rows):
    """A serving step as a graph: the same bits as without one, with new rows in every replay."""
    torch, ssgd, lowbit_block = env
    model = lowbit_block.GatedBlocks(640, 900, 2, seed=6)
    model.quantize_weights()
    x = torch.randn(rows, 640, device="cuda").to(torch.bfloat16)
    # what a program takes that goes on from 8-bit rows, or from rows as they are
    def step():
        out = model.answer(x)
        h = ssgd.mx_gated(out, model.q_up[0][0], output="fp8")
        return out, ssgd.mx_dense(h, model.q_down[0][0], bias=model.bias[0], activation="gelu", residual=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        x.copy_(torch.randn(rows, 640, device="cuda"))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
