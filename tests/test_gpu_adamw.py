"""AdamW over many tensors against its formulas in 64 bits, through the public entry points."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24          # half a unit in the last place of fp32, relative


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2003_10579_amd import ssgd
    assert torch.cuda.is_available(), "this test needs the GPU"
    ssgd.lib()
    return torch, ssgd


def _mix(x):
    x = x ^ (x >> np.uint64(16)); x = (x * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(15)); x = (x * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def _dither(total, seed, t):
    u = np.uint64
    with np.errstate(over="ignore"):
        key = _mix(u(seed >> 32) ^ _mix(u(seed & 0xFFFFFFFF) ^ _mix(u(t))))
        h = _mix(np.arange(total, dtype=np.uint64) ^ key)
    return h & u(0xFFFF), h >> u(16)


def _places(sizes):
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // 128) * 128
    return out, at


class Reference:
    """The update in 64 bits on flat arrays, from given moments."""

    def __init__(self, sizes, p, betas, eps, decay, max_norm):
        self.sizes, self.betas, self.eps, self.max_norm = sizes, betas, eps, max_norm
        self.places, self.total = _places(sizes)
        self.p = self.flat(p)
        self.decay = np.zeros(self.total)
        for n, at, d in zip(sizes, self.places, decay):
            self.decay[at:at + n] = d

    def flat(self, parts):
        out = np.zeros(self.total)
        for n, at, x in zip(self.sizes, self.places, parts):
            out[at:at + n] = x
        return out

    def after(self, m, v, lr, t):
        """The parameters of an update whose new moments are these."""
        b1, b2 = self.betas
        self.update = lr / (1 - b1 ** t) * m / (np.sqrt(v / (1 - b2 ** t)) + self.eps)
        return self.p - lr * self.decay * self.p - self.update

    def step(self, grads, m, v, lr, t):
        g = self.flat(grads)
        b1, b2 = self.betas
        norm = math.sqrt(float(np.dot(g, g)))
        c = min(1.0, self.max_norm / (norm + 1e-6)) if self.max_norm else 1.0
        # the terms of the first moment can cancel: its error, and with it the update's, goes by their magnitudes
        self.terms = b1 * np.abs(m) + (1 - b1) * np.abs(c * g)
        m = b1 * m + (1 - b1) * c * g
        v = b2 * v + (1 - b2) * (c * g) ** 2
        self.p = self.after(m, v, lr, t)
        return m, v, norm


def _host(x):
    return x.float().cpu().numpy().astype(np.float64)


SIZES = [[1], [127], [128], [129], [8192], [8193], [3, 0, 5000, 1, 40000, 129], [0], [17] * 500, [3072 * 512, 512, 5120, 10]]


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [0.0, 1.0])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_three_steps_with_moments_in_32_bits(env, sizes, max_norm, grad, offset):
    torch, ssgd = env
    g = torch.Generator().manual_seed(len(sizes) + sizes[0])
    # offset 1: no tensor begins at a multiple of 16 bytes
    cut = lambda x: x[offset:]  # noqa: E731
    ps = [cut(torch.randn(n + offset, generator=g).cuda()) for n in sizes]
    copies = [None if k % 3 == 2 else cut(torch.full((n + offset,), -7.0, dtype=torch.bfloat16, device="cuda")) for k, n in enumerate(sizes)]
    decay = [0.1 if k % 2 == 0 else 0.0 for k in range(len(sizes))]
    ref = Reference(sizes, [_host(p) for p in ps], (0.9, 0.999), 1e-8, decay, max_norm)
    opt = ssgd.AdamW(ps, weight_decay=decay, max_norm=max_norm, copies=copies)
    assert opt.m.numel() == ref.total
    assert not opt.m.any() and not opt.v.any()
    for t in range(1, 4):
        kind = torch.float32 if grad == "f32" else torch.bfloat16
        grads = [cut((torch.randn(n + offset, generator=g) * 0.1).to(kind).cuda()) for n in sizes]
        before = ref.p = ref.flat([_host(p) for p in ps])
        # each step from the moments that the kernel left: those of earlier steps can be far larger than what remains of them
        m, v, norm = ref.step([_host(x) for x in grads], _host(opt.m), _host(opt.v), 0.01, t)
        opt.step(grads, 0.01)
        got = ref.flat([_host(p) for p in ps])
        # the parameters against those that the kernel's own new moments give; the moments by themselves below
        ref.p = before
        ref.p = ref.after(_host(opt.m), _host(opt.v), 0.01, t)
        # a few roundings of the parameter, of the update (rate, moments, root, quotient) and of the moments themselves
        assert np.all(np.abs(got - ref.p) <= 8 * t * ULP * (np.abs(before) + np.abs(ref.update)) + 32 * t * ULP * np.abs(ref.update) + 1e-30)
        size = np.abs(ref.flat([_host(x) for x in grads]))
        assert np.all(np.abs(_host(opt.m) - m) <= 8 * t * ULP * (np.abs(m) + size))
        assert np.all(np.abs(_host(opt.v) - v) <= 8 * t * ULP * (v + size ** 2))
        if max_norm:
            assert abs(float(opt.grad_norm) - norm) <= 4 * ULP * norm
        for p, c in zip(ps, copies):
            if c is not None:
                assert torch.equal(c, p.to(torch.bfloat16))
    assert opt.t == 3
    opt.close()


@pytest.mark.parametrize("sizes", [[1], [128], [3, 0, 5000, 1, 40000, 129], [17] * 400], ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_moments_in_8_bits_round_as_defined(env, sizes, grad):
    torch, ssgd = env
    g = torch.Generator().manual_seed(7)
    seed = 0x123456789ABCDEF
    ps = [torch.randn(n, generator=g).cuda() for n in sizes]
    ref = Reference(sizes, [_host(p) for p in ps], (0.9, 0.999), 1e-8, [0.01] * len(sizes), 1.0)
    opt = ssgd.AdamW(ps, max_norm=1.0, state_bits=8, seed=seed)
    for t in range(1, 5):
        kind = torch.float32 if grad == "f32" else torch.bfloat16
        grads = [(torch.randn(n, generator=g) * torch.exp(3 * torch.randn(n, generator=g))).to(kind).cuda() for n in sizes]
        m0 = _host(opt.m) * np.repeat(_host(opt.m_scale), 128)
        r0 = _host(opt.v) * np.repeat(_host(opt.v_scale), 128)
        before = ref.p = ref.flat([_host(p) for p in ps])
        m, v, norm = ref.step([_host(x) for x in grads], m0, r0 ** 2, 0.01, t)
        opt.step(grads, 0.01)
        # the parameters are those of the moments before they are rounded
        got = ref.flat([_host(p) for p in ps])
        update = 0.01 / (1 - 0.9 ** t) * ref.terms / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
        assert np.all(np.abs(got - ref.p) <= 8 * ULP * (np.abs(before) + np.abs(ref.update)) + 32 * ULP * update + 1e-30)
        for x, q, scale, u, floor in ((m, opt.m, opt.m_scale, _dither(ref.total, seed, t)[0], False),
                                      (np.sqrt(v), opt.v, opt.v_scale, _dither(ref.total, seed, t)[1], True)):
            q, scale = _host(q), _host(scale)
            amax = np.abs(x).reshape(-1, 128).max(1)
            assert np.all(np.abs(scale - amax / 448) <= 16 * ULP * amax / 448)
            s = np.repeat(amax / 448, 128)
            a = np.where(s > 0, np.abs(x) / np.where(s > 0, s, 1), 0)
            step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -6) - 3)
            place = a / step + u.astype(np.float64) / 65536
            n = np.floor(place)
            if floor:
                n = np.where(a > 0, np.maximum(n, 1), n)
            want = np.minimum(n * step, 448)
            # fp32 carries the place to 1e-5 of a step; nearer than that to the threshold either neighbour is right
            clear = (np.abs(place - np.round(place)) > 1e-4) & (np.abs(a / step - np.round(a / step)) > 1e-4)
            assert np.all((np.abs(q) == want)[clear])
            assert np.all(np.abs(np.abs(q) - a) <= step * 1.001)
            assert np.all((np.sign(q) == np.sign(x)) | (q == 0))
    opt.close()


def test_stochastic_rounding_follows_an_average_that_nearest_rounding_would_stop(env):
    """With a constant gradient sqrt(v / (1 - beta2^t)) is its magnitude at every t; the mean over elements of what 8 bits hold has to
    follow.  One element's root walks with steps of up to 1/8 of it; the mean over 65536 of them is held to 5 %."""
    torch, ssgd = env
    n = 65536
    p = torch.zeros(n, device="cuda")
    opt = ssgd.AdamW([p], state_bits=8, seed=3, weight_decay=0.0)
    g = torch.full((n,), 0.5, device="cuda")
    g[::128] = 8.0            # the largest of each block sets its scale
    for t in range(1, 401):
        opt.step([g], 0.0)
    root = (_host(opt.v) * np.repeat(_host(opt.v_scale), 128)).reshape(-1, 128)[:, 1:]
    want = 0.5 * math.sqrt(1 - 0.999 ** 400)
    assert abs(root.mean() / want - 1) < 0.05
    mean = (_host(opt.m) * np.repeat(_host(opt.m_scale), 128)).reshape(-1, 128)[:, 1:]
    assert abs(mean.mean() / 0.5 - 1) < 0.01
    opt.close()


def test_infinities_and_nan_follow_the_formulas(env):
    torch, ssgd = env
    for bits in (32, 8):
        p = torch.ones(384, device="cuda")
        opt = ssgd.AdamW([p], state_bits=bits, weight_decay=0.0)
        g = torch.full((384,), 0.25, device="cuda")
        g[5], g[130] = float("nan"), float("inf")
        opt.step([g], 0.1)
        x = p.cpu()
        assert torch.isnan(x[5]) and torch.isnan(x[130])          # inf / inf
        assert torch.isfinite(x).sum() == 382 and torch.allclose(x[[0, 131, 383]], torch.tensor(0.9), atol=1e-6)
        opt.step([torch.full((384,), 0.25, device="cuda")], 0.1)
        x = p.cpu()
        if bits == 32:
            assert torch.isfinite(x).sum() == 382
        else:
            assert torch.isnan(x[:256]).all() and torch.isfinite(x[256:]).all()     # the blocks with a NaN are NaN
        opt.close()
    # a norm that is no number makes every element NaN, one that is infinite zero times the gradient
    p = torch.ones(300, device="cuda")
    opt = ssgd.AdamW([p], max_norm=1.0)
    g = torch.zeros(300, device="cuda")
    g[7] = float("nan")
    opt.step([g], 0.1)
    assert torch.isnan(opt.grad_norm).all() and torch.isnan(p).all()
    opt.close()
    # squares past the range of fp32 are still added
    p = torch.ones(300, device="cuda")
    opt = ssgd.AdamW([p], max_norm=1.0)
    opt.step([torch.full((300,), 1e25, device="cuda")], 0.1)
    assert abs(float(opt.grad_norm) / (1e25 * math.sqrt(300)) - 1) < 1e-6 and torch.isfinite(p).all()
    opt.close()


def test_nothing_is_written_beside_the_tensors(env):
    torch, ssgd = env
    for bits in (32, 8):
        for n in (1, 5, 127, 8191, 8193):
            room = torch.full((n + 64,), 3.0, device="cuda")
            copy = torch.full((n + 64,), 3.0, device="cuda", dtype=torch.bfloat16)
            opt = ssgd.AdamW([room[32:32 + n]], state_bits=bits, copies=[copy[32:32 + n]])
            opt.step([torch.ones(n, device="cuda")], 0.1)
            assert torch.all(room[:32] == 3) and torch.all(room[32 + n:] == 3) and torch.all(room[32:32 + n] != 3)
            assert torch.all(copy[:32] == 3) and torch.all(copy[32 + n:] == 3)
            assert torch.all(opt.m.float()[n:] == 0) and torch.all(opt.v.float()[n:] == 0)
            opt.close()


def test_another_stream_and_a_replayed_graph_give_the_same(env):
    torch, ssgd = env
    def fresh():
        g = torch.Generator().manual_seed(2)
        p = [torch.randn(n, generator=g).cuda() for n in (70000, 33)]
        return p, [torch.randn(n, generator=g).cuda() for n in (70000, 33)], ssgd.AdamW(p, max_norm=1.0, state_bits=8)
    p, g, opt = fresh()
    for _ in range(2):
        opt.step(g, 0.1)
    want = [x.clone() for x in p]
    p, g, opt2 = fresh()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(2):
            opt2.step(g, 0.1)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, p))
    # capture: the graph repeats update 1 (its number is an argument), so replays from the same state agree
    p, g, opt3 = fresh()
    keep = [x.clone() for x in p] + [opt3.m.clone(), opt3.v.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt3.step(g, 0.1)
    results = []
    for _ in range(3):
        for x, y in zip(p + [opt3.m, opt3.v], keep):
            x.copy_(y)
        opt3.m_scale.zero_(); opt3.v_scale.zero_()
        graph.replay()
        torch.cuda.synchronize()
        results.append([x.clone() for x in p])
    p, g, opt4 = fresh()
    opt4.step(g, 0.1)
    assert all(torch.equal(a, b) for r in results for a, b in zip(r, p))
    for o in (opt, opt2, opt3, opt4):
        o.close()


def test_refusals(env):
    torch, ssgd = env
    p = torch.zeros(10, device="cuda")
    for params, more in (([], {}), ([p.cpu()], {}), ([p.double()], {}), ([torch.zeros(4, 4, device="cuda").t()[1:]], {}), ([p], dict(copies=[p])),
                         ([p], dict(copies=[])), ([p], dict(weight_decay=[0.1, 0.2])), ([p], dict(state_bits=16)), ([p], dict(betas=(1.0, 0.9))),
                         ([p], dict(eps=0.0)), ([p], dict(max_norm=-1.0))):
        with pytest.raises(ssgd.SsgdError) as e:
            ssgd.AdamW(params, **more)
        assert e.value.status == ssgd.EINVAL
    opt = ssgd.AdamW([p])
    for grads in ([], [p, p], [p[:5]], [p.double()], [p.cpu()], [torch.zeros(20, device="cuda")[::2]]):
        with pytest.raises(ssgd.SsgdError) as e:
            opt.step(grads, 0.1)
        assert e.value.status == ssgd.EINVAL
    with pytest.raises(ssgd.SsgdError):
        opt.step([p], float("nan"))
    assert opt.t == 0
    opt.close()
    with pytest.raises(ssgd.SsgdError):
        opt.step([p], 0.1)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_checkpoint_that_is_assigned(env, bits):
    """Moments that a program assigns are what the next step uses: two steps, and one step from the stored state of the first, agree."""
    torch, ssgd = env
    g = torch.Generator().manual_seed(bits)
    start, grads = torch.randn(700, generator=g).cuda(), [torch.randn(700, generator=g).cuda() for _ in range(2)]
    p = start.clone()
    opt = ssgd.AdamW([p], state_bits=bits, seed=9)
    opt.step(grads[:1], 0.1)
    names = ("m", "v", "m_scale", "v_scale")
    stored = {k: None if getattr(opt, k) is None else getattr(opt, k).clone() for k in names}
    q = p.clone()
    opt.step(grads[1:], 0.1)
    other = ssgd.AdamW([q], state_bits=bits, seed=9)
    for k in names:
        setattr(other, k, stored[k])
    other.t = 1
    del stored
    other.step(grads[1:], 0.1)
    assert torch.equal(p, q) and torch.equal(opt.m.float(), other.m.float()) and torch.equal(opt.v.float(), other.v.float())
    opt.close()
    other.close()


def test_a_moved_parameter_is_refused(env):
    torch, ssgd = env
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    opt = ssgd.AdamW([p])
    g = torch.ones(300, device="cuda")
    opt.step([g], 0.1)
    before = p.data
    p.data = before.clone()
    with pytest.raises(ssgd.SsgdError) as e:
        opt.step([g], 0.1)
    assert e.value.status == ssgd.EINVAL and opt.t == 1
    p.data = before
    opt.step([g], 0.1)
    assert opt.t == 2
    opt.close()


def test_torch_sees_that_a_step_has_changed_the_parameters(env):
    """What autograd has kept of a parameter or its copy for a backward pass is out of date after a step: torch has to refuse it."""
    torch, ssgd = env
    p, frozen = torch.nn.Parameter(torch.ones(300, device="cuda")), torch.ones(50, device="cuda")
    copy = torch.ones(300, device="cuda", dtype=torch.bfloat16)
    with torch.inference_mode():
        apart = torch.ones(20, device="cuda")           # (has no counter)
    opt = ssgd.AdamW([p, frozen, apart], copies=[copy, None, None])
    x = torch.ones(300, device="cuda", requires_grad=True)
    before = [t._version for t in (p, frozen, copy)]
    loss = (x * p).sum()
    opt.step([torch.ones_like(t) for t in (p, frozen, apart)], 0.1)
    assert all(t._version > b for t, b in zip((p, frozen, copy), before))
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    assert torch.all(p < 1) and torch.all(apart < 1)
    opt.close()
