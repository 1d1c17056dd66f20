"""The operators of a gated feed-forward block in few bits that the framework's speed is judged on, through the public entry
points of `paper_2003_10579_amd.ssgd`, beside their plain form in elementary torch operations.

Families (the `family` key of a case):

  dense     rows times a weight matrix in 4 bits that is laid out once, with bias, activation and residual in the product's
            epilogue; the result as a matrix or in 8 bits for the next product, and what the backward pass needs of it kept.
  gated     both projections of a gated feed-forward block, its activation and their product: the weight's rows are gate and
            up in turn, h[c] = act(p[2 c]) p[2 c + 1].
  backward  what lies between the products of a backward pass: the gradient of the activation (gated or not) from a
            checkpoint, in 8 bits along its rows and along its columns, with the bias's gradient, the activation's output
            again along its columns, and the checkpoint of the product's input along its columns.
  norms     the norm behind a block, its gate and the scaled residual, and the norm in front of the next block; in training
            the gradients.

Microscaled matrices share a scale per 32 columns; the sizes go from single rows to generic wide blocks.
"""
import math

import torch

own = False

BLOCK = 32                    # columns per scale
EPS = 1e-6
SCALE = 0.75                  # of the residual


def listed():
    return [
        # the down projection of a serving step of one token, with the residual
        dict(name="dense one row", family="dense", M=1, N=4096, K=11008, x="bf16", act="none", bias=False, residual=True, out="bf16", keep="none"),
        # a layer of a ragged training step: bias and relu, in 8 bits for the next layer, the sums kept in 8 bits
        dict(name="dense ragged", family="dense", M=1027, N=1500, K=2100, x="bf16", act="relu", bias=True, residual=False, out="fp8", keep="fp8"),
        # a long prompt: everything in the epilogue
        dict(name="dense large", family="dense", M=8192, N=8192, K=8192, x="fp8", act="gelu", bias=True, residual=True, out="bf16", keep="none"),
        # both projections of a serving step of one token
        dict(name="gated one row", family="gated", M=1, H=11008, K=4096, x="bf16", act="silu", out="bf16", keep="none"),
        # a serving step of a ragged batch
        dict(name="gated 37 rows", family="gated", M=37, H=3000, K=5000, x="fp8", act="gelu", out="bf16", keep="none"),
        # a training step's block
        dict(name="gated train", family="gated", M=8192, H=8192, K=4096, x="fp8", act="silu", out="fp8", keep="fp8"),
        # a small ragged step of a layer with a bias, its sums kept as they are
        dict(name="backward dense", family="backward", M=129, H=777, D=300, gated=False, act="gelu", pre="bf16", dtype="bf16", bias=True, back="fp4"),
        # a ragged step of a gated block from 8-bit checkpoints
        dict(name="backward ragged", family="backward", M=1001, H=1537, D=1100, gated=True, act="gelu", pre="fp8", dtype="f32", bias=False, back="fp4"),
        # a training step's block from 8-bit checkpoints
        dict(name="backward train", family="backward", M=8192, H=8192, D=4096, gated=True, act="silu", pre="fp8", dtype="bf16", bias=False, back="fp8"),
        # one row of a serving step, in 8 bits for the product behind it
        dict(name="norms one row", family="norms", rows=1, d=4096, dtype="bf16", out="fp8", gate="column", groups=1, train=False),
        # ragged fp32 rows of a training step, a gate for each of 23 samples
        dict(name="norms ragged", family="norms", rows=2047, d=1537, dtype="f32", out="same", gate="group", groups=23, train=True),
        # a long batch of a training step
        dict(name="norms train", family="norms", rows=16384, d=4096, dtype="bf16", out="fp8", gate="group", groups=8, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    fam = rng.choice(["dense", "dense", "gated", "gated", "backward", "backward", "norms", "norms"])
    acts = ["relu", "gelu", "silu"]
    # (a result in 32 bits is more than one in 16 where the rows have 4)
    x = rng.choice(["bf16", "f32", "fp8", "fp4"])
    out = rng.choice(["f32" if x == "fp4" else "bf16", "bf16", "fp8"])
    if fam == "dense":
        return dict(family=fam, M=_log_int(rng, 1, 8192), N=_log_int(rng, 64, 8192), K=_log_int(rng, 64, 8192), x=x, act=rng.choice(["none"] + acts),
                    bias=rng.choice([True, False]), residual=rng.choice([True, False]), out=out, keep=rng.choice(["none", "same", "fp8"]))
    if fam == "gated":
        return dict(family=fam, M=_log_int(rng, 1, 8192), H=_log_int(rng, 32, 8192), K=_log_int(rng, 64, 4096), x=x, act=rng.choice(acts), out=out,
                    keep=rng.choice(["none", "same", "fp8"]))
    if fam == "backward":
        gated = rng.choice([True, False])
        return dict(family=fam, M=_log_int(rng, 1, 8192), H=_log_int(rng, 16, 8192), D=_log_int(rng, 64, 4096), gated=gated, act=rng.choice(acts),
                    pre=rng.choice(["bf16", "f32", "fp8"]), dtype=rng.choice(["bf16", "f32"]), bias=not gated, back=rng.choice(["fp4", "fp8"]))
    d = _log_int(rng, 64, 16384)
    gate = rng.choice(["none", "column", "group"])
    groups = _log_int(rng, 1, 64) if gate == "group" else 1
    return dict(family=fam, rows=groups * _log_int(rng, 1, max(1, min(16384, 64000000 // d) // groups)), d=d, dtype=rng.choice(["bf16", "f32"]),
                out=rng.choice(["fp8", "same"]), gate=gate, groups=groups, train=rng.choice([True, False]))


# ------------------------------------------------------------------------------------------------------------- state

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _heavy(shape, g):
    """Values of layers in training: normal with a few entries that are far larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x * (1.0 + 20.0 * (torch.rand(shape, generator=g, device="cuda") < 0.001))


def _given(x, kind):
    """A matrix that a program has in hand: of a plain type, or microscaled."""
    if kind in _TYPES:
        return x.to(_TYPES[kind])
    if own:
        from paper_2003_10579_amd import ssgd
        return ssgd.mx_quantize(x, kind)
    q, scale = _quantize(x, kind)
    return q.to(torch.float8_e4m3fn), scale, x.shape[1]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": case}
    fam = case["family"]
    if fam in ("dense", "gated"):
        M, K = case["M"], case["K"]
        N = case["N"] if fam == "dense" else 2 * case["H"]
        s["x"] = _given(_heavy((M, K), g), case["x"])
        s["w"] = _given(normal(N, K) / math.sqrt(K), "fp4")
        if fam == "dense":
            s["bias"] = 0.2 * normal(N) if case["bias"] else None
            s["residual"] = normal(M, N).to(_TYPES["f32" if case["out"] == "f32" else "bf16"]) if case["residual"] else None
    elif fam == "backward":
        M, H = case["M"], case["H"]
        s["dy"] = (_heavy((M, H), g) * 1e-3).to(_TYPES[case["dtype"]])
        s["pre"] = _given(1.5 * normal(M, 2 * H if case["gated"] else H), case["pre"])
        s["y"] = _given(_heavy((M, case["D"]), g), "fp8")
    else:
        shape, t = (case["rows"], case["d"]), _TYPES[case["dtype"]]
        s["o"], s["s"] = (3.0 * _heavy(shape, g)).to(t), normal(*shape).to(t)
        s["w_post"], s["w"] = 1.0 + 0.1 * normal(case["d"]), 1.0 + 0.1 * normal(case["d"])
        s["gate"] = None if case["gate"] == "none" else 0.5 * normal(case["d"]) if case["gate"] == "column" else 0.5 * normal(case["groups"], case["d"])
        if case["train"]:
            s["dy"], s["dsum"] = normal(*shape).to(t), normal(*shape).to(t)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms

def _power(e):
    """2^e in 32 bits, -127 <= e <= 127, from its bits: a power function may be off in the last place."""
    return torch.where(e >= -126, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantize(x, fmt):
    """Per 32 columns the exponent of the largest magnitude less that of the format's largest value, and the values at
    that scale rounded to the nearest one of the format (ties to the even code), the largest where they are past it."""
    top, most, least, digits = {"fp4": (2, 6.0, 0, 1), "fp8": (8, 448.0, -6, 3)}[fmt]
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % BLOCK)).view(x.shape[0], -1, BLOCK)
    amax = x.abs().amax(2, keepdim=True)
    e = torch.frexp(amax)[1] - 1 - top
    e = torch.where(amax > 0, e, -127).clamp(-127, 127)
    a = (x.abs() * _power(-e)).clamp(max=most)
    step = _power((torch.frexp(a)[1] - 1).clamp(min=least) - digits)
    q = torch.round(a / step) * step * torch.sign(x)
    return q, (e + 127).to(torch.uint8)[:, :, 0]


def _read_back(q, scale, cols):
    return (q.float() * _power(scale.int() - 127)[:, :, None]).reshape(q.shape[0], -1)[:, :cols]


def _values(x, fmt=None):
    """What a given matrix stands for; rows of a plain type are quantised to `fmt` on the way, where there is one."""
    if isinstance(x, tuple):
        return _read_back(*x)
    return x.float() if fmt is None else _read_back(*_quantize(x, fmt), x.shape[1])


def _held(q, scale, cols):
    """An output in 8 bits as its values and scales."""
    return {"values": q.reshape(q.shape[0], -1)[:, :cols].to(torch.float8_e4m3fn), "scales": scale.view(torch.float8_e8m0fnu)}


def _eight(x):
    return _held(*_quantize(x, "fp8"), x.shape[1])


def _columns(x, fmt):
    """An output along the columns of x: 4-bit values times their scale are E5M2 numbers."""
    if fmt == "fp8":
        return _eight(x.t())
    return _read_back(*_quantize(x.t(), "fp4"), x.shape[0]).to(torch.float8_e5m2)


def _act(x, act):
    if act == "relu":
        return torch.where(x > 0, x, 0.0)
    if act == "gelu":
        return 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    return x / (1.0 + torch.exp(-x)) if act == "silu" else x


def _slope(x, act):
    if act == "relu":
        return torch.where(x > 0, 1.0, 0.0)
    if act == "gelu":
        return 0.5 * torch.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * math.sqrt(0.5 / math.pi)
    sigma = 1.0 / (1.0 + torch.exp(-x))
    return sigma * (1.0 + x * (1.0 - sigma))


def _result(x, kind):
    return _eight(x) if kind == "fp8" else x.to(_TYPES[kind])


def _kept(out, p, case):
    if case["keep"] != "none":
        out["kept"] = _result(p, "fp8" if case["keep"] == "fp8" else "f32" if case["out"] == "f32" else "bf16")
    return out


def _plain_norms(s):
    case = s["case"]
    t = s["o"].dtype
    # (the sum in 64 bits: what it is rounded to is next to a border now and then, and all that follows goes by it)
    o = s["o"].double()
    rstd_o = torch.rsqrt(o.square().mean(1, keepdim=True) + EPS)
    gate = 1.0 if s["gate"] is None else s["gate"].view(-1, case["d"]).repeat_interleave(case["rows"] // case["groups"], 0)
    total = (SCALE * s["s"].double() + gate * (o * rstd_o * s["w_post"])).to(t)
    o, rstd_o = s["o"].float(), rstd_o.float()
    ohat = o * rstd_o
    f = total.float()
    rstd = torch.rsqrt(f.square().mean(1, keepdim=True) + EPS)
    shat = f * rstd
    y = shat * s["w"]
    out = {"sum": total, "rstd_o": rstd_o[:, 0], "rstd": rstd[:, 0], "y": _eight(y) if case["out"] == "fp8" else y.to(t)}
    if case["train"]:
        dy = s["dy"].float()
        gw = dy * s["w"]
        grad = rstd * (gw - shat * (gw * shat).mean(1, keepdim=True)) + s["dsum"].float()
        gp = grad * gate * s["w_post"]
        out["do"] = (rstd_o * (gp - ohat * (gp * ohat).mean(1, keepdim=True))).to(t)
        out["ds"] = (SCALE * grad).to(t)
        out["dw_post"], out["dw"] = (grad * gate * ohat).sum(0), (dy * shat).sum(0)
        if s["gate"] is not None:
            out["dgate"] = (grad * ohat * s["w_post"]).view(case["groups"], -1, case["d"]).sum(1).view(s["gate"].shape)
    return out


def _plain(s):
    case = s["case"]
    fam = case["family"]
    if fam == "norms":
        return _plain_norms(s)
    if fam == "backward":
        pre, dy = _values(s["pre"]), s["dy"].float()
        if case["gated"]:
            gate, up = pre[:, 0::2], pre[:, 1::2]
            h = _act(gate, case["act"])
            d = torch.stack((dy * up * _slope(gate, case["act"]), dy * h), 2).reshape(case["M"], -1)
            h = h * up
        else:
            h, d = _act(pre, case["act"]), dy * _slope(pre, case["act"])
        out = {"rows": _eight(d), "cols": _eight(d.t()), "h": _columns(h, case["back"]), "y": _columns(_values(s["y"]), case["back"])}
        if case["bias"]:
            out["dbias"] = d.sum(0)
        return out
    p = torch.matmul(_values(s["x"], "fp8"), _values(s["w"]).t())
    if fam == "gated":
        return _kept({"h": _result(_act(p[:, 0::2], case["act"]) * p[:, 1::2], case["out"])}, p, case)
    if case["bias"]:
        p = p + s["bias"]
    y = _act(p, case["act"])
    if case["residual"]:
        y = s["residual"].float() + y
    return _kept({"y": _result(y, case["out"])}, p, case)


# --------------------------------------------------------------------------------------------- the framework's kernels

def _shown(q):
    """An MxTensor as its values and scales, without the padding; from 4 bits the values times their scale."""
    from paper_2003_10579_amd import ssgd
    if not isinstance(q, ssgd.MxTensor):
        return q
    if q.format == "fp4":
        return ssgd.mx_dequantize(q, torch.bfloat16).to(torch.float8_e5m2)
    return {"values": q.values.view(torch.float8_e4m3fn)[:, :q.shape[1]], "scales": q.scales.view(torch.float8_e8m0fnu)[:, :-(-q.shape[1] // BLOCK)]}


def _kernels(s):
    from paper_2003_10579_amd import ssgd
    case = s["case"]
    fam = case["family"]
    if fam == "norms":
        y, total, rstd_o, rstd = ssgd.block_norm(s["o"], s["s"], s["w_post"], s["w"], gate=s["gate"], scale=SCALE, eps=EPS, output="fp8" if case["out"] == "fp8" else None)
        out = {"sum": total, "rstd_o": rstd_o, "rstd": rstd, "y": _shown(y)}
        if case["train"]:
            out["do"], out["ds"], out["dw_post"], out["dw"], dgate = ssgd.block_norm_backward(s["dy"], s["o"], total, s["w_post"], s["w"], rstd_o, rstd, gate=s["gate"], scale=SCALE,
                                                                                              dsum=s["dsum"])
            if dgate is not None:
                out["dgate"] = dgate
        return out
    if fam == "backward":
        if case["gated"]:
            rows, cols, h = ssgd.mx_gated_backward(s["dy"], s["pre"], case["act"], hidden=case["back"])
            out = {}
        else:
            rows, cols, h, dbias = ssgd.mx_dense_backward(s["dy"], s["pre"], case["act"], hidden=case["back"])
            out = {"dbias": dbias}
        return dict(out, rows=_shown(rows), cols=_shown(cols), h=_shown(h), y=_shown(ssgd.mx_transpose(s["y"], case["back"])))
    keep = None if case["keep"] == "none" else case["keep"]
    how = {"output": "fp8"} if case["out"] == "fp8" else {"dtype": _TYPES[case["out"]]}
    if keep == "same" and case["out"] == "fp8":
        how["dtype"] = torch.bfloat16
    if fam == "gated":
        y = ssgd.mx_gated(s["x"], s["w"], case["act"], keep=keep, **how)
    else:
        y = ssgd.mx_dense(s["x"], s["w"], bias=s["bias"], activation=None if case["act"] == "none" else case["act"], residual=s["residual"], keep=keep, **how)
    name = "h" if fam == "gated" else "y"
    return {name: _shown(y)} if keep is None else {name: _shown(y[0]), "kept": _shown(y[1])}


def run(s):
    return _kernels(s) if own else _plain(s)


# ------------------------------------------------------------------------------------------------------- in 64 bits

_MAGNITUDES = {"fp4": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0],
               "fp8": [c % 8 * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)]}


def _exact_mx(x, fmt):
    """(values, scale) in 64 bits, from the table of the format's magnitudes and the middles between them."""
    table = torch.tensor(_MAGNITUDES[fmt], dtype=torch.float64, device=x.device)
    middles = (table[1:] + table[:-1]) / 2
    rows, cols = x.shape
    wide = torch.zeros(rows, -(-cols // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    wide[:, :cols] = x
    b = wide.reshape(rows, -1, BLOCK)
    largest = b.abs().max(2).values
    # the exponent field of a 64-bit number is the whole part of its logarithm
    power = torch.where(largest > 0, (largest.view(torch.int64) >> 52) - 1023 - {"fp4": 2, "fp8": 8}[fmt], -127).clamp(-127, 127)
    scale = ((power + 1023) << 52).view(torch.float64)
    scaled = (b.abs() / scale[:, :, None]).contiguous()
    low, high = torch.bucketize(scaled, middles), torch.bucketize(scaled, middles, right=True)
    code = torch.where(low % 2 == 0, low, high)
    return (table[code] * torch.where(b < 0, -1.0, 1.0)).reshape(rows, -1)[:, :cols], scale


def _exact_values(x, fmt):
    """What a microscaled matrix of x stands for."""
    q, scale = _exact_mx(x, fmt)
    return q * scale.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _exact_given(x, fmt="fp8"):
    """The same for a given matrix: an inverse of the form it is given in, or its quantisation."""
    if not isinstance(x, tuple):
        return _exact_values(x.double(), fmt) if fmt else x.double()
    q, scale, cols = x
    return (q.double() * torch.exp2(scale.double() - 127)[:, :, None]).flatten(1)[:, :cols]


def _exact_eight(x):
    q, scale = _exact_mx(x, "fp8")
    return {"values": q, "scales": scale}


def _exact_columns(x, fmt):
    return _exact_eight(x.t()) if fmt == "fp8" else _exact_values(x.t(), "fp4")


def _phi(x):
    return (1 + torch.special.erf(x / 2 ** 0.5)) / 2


def _exact_act(x, act):
    return {"none": lambda: x, "relu": lambda: x.clamp(min=0), "gelu": lambda: x * _phi(x), "silu": lambda: x * torch.sigmoid(x)}[act]()


def _exact_slope(x, act):
    if act == "relu":
        return (x > 0).double()
    if act == "gelu":
        return _phi(x) + x * torch.exp(-x * x / 2) / (2 * math.pi) ** 0.5
    sigma = torch.sigmoid(x)
    return sigma + x * sigma * torch.sigmoid(-x)


def _exact_norms(case, s):
    o = s["o"].double()
    inv_o = 1 / ((o * o).sum(1, keepdim=True) / case["d"] + EPS) ** 0.5
    post, w = s["w_post"].double(), s["w"].double()
    per = case["rows"] // case["groups"]
    gate = torch.ones(1, case["d"], dtype=torch.float64, device=o.device) if s["gate"] is None else s["gate"].double().reshape(-1, case["d"])
    wide = gate[torch.arange(case["rows"], device=o.device) // per] if gate.shape[0] > 1 else gate
    total = wide * post * (o * inv_o) + SCALE * s["s"].double()
    total = total.to(s["o"].dtype).double()
    inv = 1 / ((total * total).sum(1, keepdim=True) / case["d"] + EPS) ** 0.5
    y = total * inv * w
    out = {"sum": total, "rstd_o": inv_o[:, 0], "rstd": inv[:, 0], "y": _exact_eight(y) if case["out"] == "fp8" else y}
    if case["train"]:
        dy = s["dy"].double()
        dot = (dy * w * total).sum(1, keepdim=True) / case["d"]
        grad = inv * dy * w - inv ** 3 * dot * total + s["dsum"].double()
        through = wide * post * grad
        dot = (through * o).sum(1, keepdim=True) / case["d"]
        out["do"] = inv_o * through - inv_o ** 3 * dot * o
        out["ds"] = SCALE * grad
        out["dw"] = (dy * total * inv).sum(0)
        by_group = torch.stack([c.sum(0) for c in (grad * o * inv_o).split(per)])
        out["dw_post"] = (gate * by_group).sum(0)
        if s["gate"] is not None:
            out["dgate"] = (post * by_group).reshape(s["gate"].shape)
    return out


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    fam = case["family"]
    if fam == "norms":
        return _exact_norms(case, s)
    if fam == "backward":
        pre, dy = _exact_given(s["pre"], None), s["dy"].double()
        if case["gated"]:
            pairs = pre.unflatten(1, (-1, 2))
            a = _exact_act(pairs[:, :, 0], case["act"])
            d = torch.empty_like(pre)
            d[:, 1::2] = dy * a
            d[:, 0::2] = dy * pairs[:, :, 1] * _exact_slope(pairs[:, :, 0], case["act"])
            h = a * pairs[:, :, 1]
        else:
            h, d = _exact_act(pre, case["act"]), dy * _exact_slope(pre, case["act"])
        out = {"rows": _exact_eight(d), "cols": _exact_eight(d.t()), "h": _exact_columns(h, case["back"]), "y": _exact_columns(_exact_given(s["y"]), case["back"])}
        if case["bias"]:
            out["dbias"] = d.sum(0)
        return out
    p = _exact_given(s["x"]) @ _exact_given(s["w"]).t()
    if fam == "gated":
        y = p[:, 1::2] * _exact_act(p[:, 0::2], case["act"])
    else:
        if case["bias"]:
            p += s["bias"].double()
        y = _exact_act(p, case["act"])
        if case["residual"]:
            y = y + s["residual"].double()
    out = {"h" if fam == "gated" else "y": _exact_eight(y) if case["out"] == "fp8" else y}
    if case["keep"] != "none":
        out["kept"] = _exact_eight(p) if case["keep"] == "fp8" else p
    return out


# -------------------------------------------------------------------------------------------- what a pass cannot avoid

_BYTES = {"f32": 4.0, "bf16": 2.0, "fp8": 1 + 1 / BLOCK, "fp4": 0.5 + 1 / BLOCK}


def work(case):
    """Every input read once and every output written once; the operations of the products, and about one per byte else."""
    fam = case["family"]
    if fam == "norms":
        n, b = float(case["rows"] * case["d"]), _BYTES[case["dtype"]]
        sides = (2 if case["train"] else 1) * 4.0 * (2 * case["d"] + case["rows"] + (0 if case["gate"] == "none" else case["groups"] * case["d"]))
        return {"bytes": n * (3 * b + (_BYTES["fp8"] if case["out"] == "fp8" else b) + (6 * b if case["train"] else 0)) + sides, "flops": n * (40 if case["train"] else 14)}
    if fam == "backward":
        n, d, y = float(case["M"] * case["H"]), (2.0 if case["gated"] else 1.0), float(case["M"] * case["D"])
        return {"bytes": n * (_BYTES[case["dtype"]] + d * _BYTES[case["pre"]] + 2 * d * _BYTES["fp8"] + _BYTES[case["back"]]) + y * (_BYTES["fp8"] + _BYTES[case["back"]]), "flops": 20 * n + y}
    M, K = float(case["M"]), float(case["K"])
    N, results = (float(case["N"]), float(case["N"])) if fam == "dense" else (2.0 * case["H"], float(case["H"]))
    plain = _BYTES["f32" if case["out"] == "f32" else "bf16"]
    kept = {"none": 0.0, "same": plain, "fp8": _BYTES["fp8"]}[case["keep"]]
    beside = plain if fam == "dense" and case["residual"] else 0.0
    return {"bytes": _BYTES[case["x"]] * M * K + _BYTES["fp4"] * N * K + M * results * (_BYTES[case["out"]] + beside) + M * N * kept, "flops": 2 * M * N * K}
