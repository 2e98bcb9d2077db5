"""Performance cases of the operators around the 8-bit linears of a transformer
block: RMS norm with the residual's addition (16-bit output, or rotated and
quantized to 8 bits), rotary positions with several axes, and the 8-bit linear
with activation, gate and residual in its epilogue.

8-bit codes: a row's scale is max|x| / 127 after the rotation by Hadamard blocks
of `block` columns (in 32 bits, neighbours first), a code the rotated value times
127 / max|x|, rounded to 32 bits, to the nearest whole number, ties to even.
Weights hold the rotation and its 1 / block.

`own = False` computes every operator in elementary torch operations in 32 bits;
`own = True` makes the library's calls.
"""
import math

import torch

own = False

_TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}
_BYTES = {"float16": 2, "bfloat16": 2, "float32": 4, "none": 0}
EPS = 1e-6
THETA = 10000.0


def _lib():
    import paper_2509_24416_amd as clq
    return clq


def _norm(name, M, K, block, dtype, residual, samples=1, perm=False, weight="float16"):
    """block 0: the plain 16-bit output."""
    return dict(name=name, kind="norm8" if block else "norm", M=M, K=K, block=block, dtype=dtype, residual=residual,
                samples=samples, perm=perm, weight=weight)


def _rope(name, M, tokens, heads, axes, dtype, interleaved, norm, inverse=False, unrotated=0):
    """axes: the columns of a head that time, height and width rotate; unrotated: the head's others."""
    time, height, width = axes
    return dict(name=name, kind="rope", M=M, tokens=tokens, heads=heads, time=time, height=height, width=width,
                dtype=dtype, interleaved=interleaved, norm=norm, inverse=inverse, unrotated=unrotated)


def _linear(name, M, K, N, bits, dtype, act="none", gate=0, residual=False, bias=True, block=64):
    """gate: the samples that have a gate of their own (0: none)."""
    return dict(name=name, kind="linear", M=M, K=K, N=N, bits=bits, dtype=dtype, act=act, gate=gate,
                residual=residual, bias=bias, block=block)


def listed():
    return [
        # one token's norm ahead of its 8-bit linear: launch and latency only
        _norm("norm8_token", 1, 1152, 64, "float16", "float16"),
        # a token count that fills no tile, a residual stream in 32 bits, the swap of outlier channels
        _norm("norm8_ragged_swap", 2777, 1216, 32, "bfloat16", "float32", perm=True),
        # every token of a video step, two guidance samples with a modulation of their own
        _norm("norm8_video", 43200, 1152, 64, "float16", "float16", samples=2),
        # caption tokens of a text encoder's width under guidance batch 2, no residual
        _norm("norm_caption", 600, 4096, 0, "bfloat16", "none"),
        # a 1024-pixel image's tokens at an MLP's width, the residual added
        _norm("norm_image", 8192, 4608, 0, "bfloat16", "bfloat16", samples=2),
        # queries and keys of one new token
        _rope("rope_token", 2, 1, 32, (24, 24, 24), "float16", True, False),
        # queries and keys of a video step: 16 frames of 30 x 45 patches, guidance batch 2
        _rope("rope_video", 43200, 21600, 32, (24, 24, 24), "float16", True, False),
        # joint image and caption tokens, heads normed, halves of a head paired
        _rope("rope_norm_image", 4608, 4608, 48, (16, 56, 56), "bfloat16", False, True),
        # one token through an MLP's first layer: the weights are read once for a single row
        _linear("linear_token", 1, 1152, 4608, 8, "float16", act="gelu"),
        # sizes that fill no tile, 4-bit weights, everything in the epilogue
        _linear("linear_ragged", 777, 1216, 1000, 4, "bfloat16", act="silu", gate=1, residual=True, block=32),
        # the MLP's second layer over a video step: gated into the residual stream
        _linear("linear_video", 43200, 4608, 1152, 8, "float16", gate=2, residual=True),
        # the whole MLP half of an image transformer's block, norm to residual
        dict(name="mlp_image", kind="mlp", M=8192, K=1152, F=4608, bits=8, dtype="float16", samples=2, block=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step):
    return max(1, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step


def draw(rng):
    kind = rng.choices(["norm8", "norm", "rope", "linear", "mlp"], [4, 3, 4, 5, 2])[0]
    block = rng.choice([32, 64, 64, 128])
    dtype = rng.choice(["float16", "bfloat16"])
    samples = rng.choice([1, 1, 2])
    rows = _log_int(rng, 1, 43200 // samples) * samples
    if kind in ("norm8", "norm"):
        K = _width(rng, 64, 8192, max(64, block)) if kind == "norm8" else _width(rng, 64, 8192, 8)
        while rows * K > 43200 * 1152:
            rows = (rows // samples // 2 + 1) * samples
        c = _norm("", rows, K, block if kind == "norm8" else 0, dtype, rng.choice([dtype, dtype, "float32", "none"]),
                  samples, kind == "norm8" and rng.random() < 0.3, rng.choice(["float16", "bfloat16", "float32", "none"]))
    elif kind == "rope":
        axes = rng.choice([(16, 24, 24), (24, 24, 24), (16, 56, 56), (32, 16, 16), (8, 12, 12), (44, 42, 42)])
        unrotated = rng.choice([0, 0, 0, 32])
        heads = rng.randint(1, 64)
        while rows * heads * (sum(axes) + unrotated) > 43200 * 32 * 72:
            rows = (rows // samples // 2 + 1) * samples
        c = _rope("", rows, rows // samples, heads, axes, dtype, rng.random() < 0.5, rng.random() < 0.5,
                  rng.random() < 0.2, unrotated)
    elif kind == "linear":
        K, N = _width(rng, 128, 4608, max(64, block)), _log_int(rng, 16, 4608)
        while rows * K * N > 43200 * 1152 * 4608 or rows * (K + N) > 43200 * 5760:
            rows = (rows // samples // 2 + 1) * samples
        c = _linear("", rows, K, N, rng.choice([4, 8, 8]), rng.choice([dtype, dtype, "float32"]),
                    rng.choice(["none", "gelu", "silu"]), rng.choice([0, samples]), rng.random() < 0.6,
                    rng.random() < 0.8, block)
    else:
        K, F = _width(rng, 128, 1152, 128), _width(rng, 256, 4608, 128)
        while rows * K * F > 43200 * 1152 * 2304:
            rows = (rows // samples // 2 + 1) * samples
        c = dict(kind=kind, M=rows, K=K, F=F, bits=rng.choice([4, 8]), dtype=dtype, samples=samples, block=block)
    c.pop("name", None)
    return c


# ---- inputs ---------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _activations(g, M, K, dtype):
    """Gaussian tokens with 1 % of the channels 20 to 100 times as large (the
    outlier channels that the rotation is there for)."""
    gain = torch.ones(K, device="cuda")
    hot = torch.randperm(K, device="cuda", generator=g)[: max(1, K // 100)]
    gain[hot] = 20.0 * 5.0 ** torch.rand(hot.numel(), device="cuda", generator=g)
    return (_normal(g, M, K) * gain).to(_TYPES[dtype])


def _stream(g, M, K, dtype):
    return (3.0 * _normal(g, M, K)).to(_TYPES[dtype])


def _modulation(g, samples, K, dtype):
    """1 + a sample's scale, [K] or [samples, K]."""
    w = 1.0 + 0.2 * _normal(g, samples, K)
    return (w if samples > 1 else w[0]).to(_TYPES[dtype])


def _weights(g, N, K, block, bits):
    """fp16 weights as a checkpoint holds them, and their codes and scales: rotated, one scale a
    channel, the rotation's 1 / block in it."""
    w = (_normal(g, N, K) / math.sqrt(K)).half()
    v = _butterflies(w.float(), 1, block)
    top, most = v.abs().amax(-1), 127.0 if bits == 8 else 7.0
    return w, _whole(v, _ratio(most, top)), _ratio(top, most) / block


def _positions(case, g):
    """Time, height and width of each token of a sample: a grid's, behind a few tokens that have none
    (a caption's, at 0); a single token is somewhere in it."""
    n = case["tokens"]
    if n == 1:
        return torch.randint(0, 4096, (1, 3), device="cuda", generator=g).to(torch.int32)
    H, W = (30, 45) if n >= 2 * 1350 else (max(1, int(math.sqrt(n))),) * 2
    i = torch.arange(n, device="cuda") - n % (H * W)
    at = torch.stack((i.div(H * W, rounding_mode="floor"), i.div(W, rounding_mode="floor") % H, i % W), -1)
    return torch.where(i.unsqueeze(-1) < 0, 0, at).to(torch.int32)


def _axes(case):
    return case["time"], case["height"], case["width"]


def _freqs(case):
    """Radians a position for each pair: an axis of d columns has theta^(-2 j / d), j = 0 .. d / 2 - 1."""
    return torch.cat([THETA ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
                      for d in _axes(case)])


def _inputs(case, seed):
    g, kind, s = _gen(seed), case["kind"], dict(case)
    M = case["M"]
    if kind in ("norm", "norm8"):
        K = case["K"]
        s["x"] = _activations(g, M, K, case["dtype"])
        s["r"] = None if case["residual"] == "none" else _stream(g, M, K, case["residual"])
        s["w"] = None if case["weight"] == "none" else _modulation(g, case["samples"], K, case["weight"])
        s["swap"] = torch.randperm(K, device="cuda", generator=g).to(torch.int32) if case["perm"] else None
    elif kind == "rope":
        D = sum(_axes(case)) + case["unrotated"]
        # queries and keys as a projection leaves them: the first columns of rows that hold the values too
        wide = _normal(g, M, case["heads"] * D + 8 * ((case["heads"] * D + 15) // 16)).to(_TYPES[case["dtype"]])
        s["x"] = wide[:, : case["heads"] * D].view(M, case["heads"], D)
        s["at"] = _positions(case, g)
        s["freqs"] = _freqs(case)
        s["w"] = _modulation(g, case["heads"], D, case["dtype"]) if case["norm"] else None
    else:
        K, N = case["K"], case.get("N", case["K"])
        if kind == "linear":
            s["x"] = _activations(g, M, K, "float16")
            s["w"], s["codes"], s["scale"] = _weights(g, N, K, case["block"], case["bits"])
            samples = case["gate"]
            s["b"] = (0.1 * _normal(g, N)).to(torch.float16) if case["bias"] else None
            s["r"] = _stream(g, M, N, case["dtype"]) if case["residual"] else None
        else:
            F, samples = case["F"], case["samples"]
            s["x"] = _activations(g, M, K, "float16")
            s["r"] = _stream(g, M, K, case["dtype"])
            s["n"] = _modulation(g, samples, K, "float16")
            s["w1"], s["codes1"], s["scale1"] = _weights(g, F, K, case["block"], case["bits"])
            s["w2"], s["codes2"], s["scale2"] = _weights(g, K, F, case["block"], case["bits"])
            s["b1"] = (0.1 * _normal(g, F)).to(torch.float16)
            s["b2"] = (0.1 * _normal(g, K)).to(torch.float16)
        s["g"] = _modulation(g, samples, N, case["dtype"]) if samples else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] in ("linear", "mlp"):
        # weights are quantized and laid out once, when a program loads them
        lib = _lib()
        quantize = lib.clq_quantize_weights8 if case["bits"] == 8 else lib.clq_quantize_weights
        for name in ("w", "w1", "w2"):
            if name in s:
                s["q" + name] = quantize(s[name], case["block"])
    return s


# ---- the plain forms --------------------------------------------------------------

def _butterflies(v, h, block):
    """Stages h, 2h, ..., block / 2 of the unnormalised Hadamard transform."""
    if h >= block:
        return v
    p = v.unflatten(-1, (-1, 2, h))
    lo, hi = p[..., 0, :], p[..., 1, :]
    return _butterflies(torch.stack((lo + hi, lo - hi), -2).flatten(-3), 2 * h, block)


def _ratio(a, b):
    """a / b rounded once to 32 bits, 0 where both scale a row of zeros."""
    a, b = torch.as_tensor(a, dtype=torch.float64), torch.as_tensor(b, dtype=torch.float64)
    return torch.where(b == 0, 0.0, a / b).float()


def _whole(v, r):
    """v times its row's r, to the nearest whole number (the product in 64 bits: it is next to a border often)."""
    return torch.round(v.double() * r.double().unsqueeze(-1)).float()


def _quantized(v, block):
    """Codes and scales of rows rotated by blocks."""
    v = _butterflies(v, 1, block)
    top = v.abs().amax(-1)
    return _whole(v, _ratio(127.0, top)), _ratio(top, 127.0)


def _by_sample(w, M):
    """[K] or [samples, K] as a row for each token."""
    w = w.float()
    return w if w.dim() == 1 else w.repeat_interleave(M // w.shape[0], 0)


def _normed(s):
    v = s["x"].float()
    v = v if s["r"] is None else v + s["r"].float()
    n = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v, n if s["w"] is None else n * _by_sample(s["w"], s["M"])


def _plain_norm(s):
    v, n = _normed(s)
    if s["kind"] == "norm8":
        codes, scale = _quantized(n if s["swap"] is None else n[:, s["swap"].long()], s["block"])
        n = codes * scale.unsqueeze(-1)
    y = {"y": n.to(s["x"].dtype)}
    return y if s["r"] is None else {**y, "sum": v.to(s["r"].dtype)}


def _plain_rope(s):
    v = s["x"].float()
    if s["w"] is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * s["w"].float()
    i = torch.arange(sum(_axes(s)) // 2, device=v.device)
    axis = (2 * i >= s["time"]).long() + (2 * i >= s["time"] + s["height"]).long()
    angle = s["at"].double()[:, axis] * s["freqs"]
    angle = angle.repeat(s["M"] // s["tokens"], 1).unsqueeze(1)
    c, d = torch.cos(angle).float(), torch.sin(angle).float()
    d = -d if s["inverse"] else d
    n = 2 * axis.numel()
    a, b = (v[..., :n:2], v[..., 1:n:2]) if s["interleaved"] else (v[..., : n // 2], v[..., n // 2:n])
    a, b = a * c - b * d, b * c + a * d
    turned = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, v[..., n:]), -1).to(s["x"].dtype)


def _activated(v, act):
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.tanh(0.7978845608028654 * (v + 0.044715 * v * v * v)))
    return v / (1.0 + torch.exp(-v)) if act == "silu" else v


def _product(codes, scale, wcodes, wscale, bias):
    y = (codes @ wcodes.t()) * scale.unsqueeze(-1) * wscale
    return y if bias is None else y + bias.float()


def _plain_linear(s):
    codes, scale = _quantized(s["x"].float(), s["block"])
    y = _activated(_product(codes, scale, s["codes"], s["scale"], s["b"]), s["act"])
    y = y if s["g"] is None else y * _by_sample(s["g"], s["M"])
    return (y if s["r"] is None else y + s["r"].float()).to(_TYPES[s["dtype"]])


def _plain_mlp(s):
    v, n = _normed({**s, "w": s["n"]})
    h = _product(*_quantized(n, s["block"]), s["codes1"], s["scale1"], s["b1"])
    h = _product(*_quantized(_activated(h, "gelu"), s["block"]), s["codes2"], s["scale2"], s["b2"])
    stream = v.to(s["r"].dtype).float()
    return (stream + _by_sample(s["g"], s["M"]) * h).to(s["r"].dtype)


def _plain(s):
    if s["kind"] in ("norm", "norm8"):
        return _plain_norm(s)
    if s["kind"] == "rope":
        return _plain_rope(s)
    return _plain_linear(s) if s["kind"] == "linear" else _plain_mlp(s)


# ---- one pass -----------------------------------------------------------------------

def run(state):
    s = state
    if not own:
        return _plain(s)
    clq = _lib()
    kind = s["kind"]
    if kind == "norm":
        y = clq.clq_rms_norm(s["x"], s["w"], s["r"], EPS)
        return {"y": y} if s["r"] is None else {"y": y[0], "sum": y[1]}
    if kind == "norm8":
        q, scale, *total = clq.clq_rms_norm_act8(s["x"], s["block"], s["w"], s["r"], EPS, perm=s["swap"])
        y = {"y": clq.clq_dequantize_act8(q, scale, s["K"], dtype=s["x"].dtype)}
        return {**y, "sum": total[0]} if total else y
    if kind == "rope":
        return clq.clq_rope_axes(s["x"], s["at"], s["freqs"], _axes(s), interleaved=s["interleaved"],
                                 inverse=s["inverse"], weight=s["w"], eps=EPS)
    if kind == "linear":
        q, scale = clq.clq_rotate_quant_act8(s["x"], s["block"])
        return clq.clq_a8_linear_act(q, scale, s["qw"], s["b"], act=s["act"], gate=s["g"], residual=s["r"],
                                     dtype=_TYPES[s["dtype"]])
    q, scale, stream = clq.clq_rms_norm_act8(s["x"], s["block"], s["n"], s["r"], EPS)
    h = clq.clq_a8_linear_act(q, scale, s["qw1"], s["b1"], act="gelu")
    q, scale = clq.clq_rotate_quant_act8(h, s["block"])
    return clq.clq_a8_linear_act(q, scale, s["qw2"], s["b2"], gate=s["g"], residual=stream, dtype=stream.dtype)


def work(case):
    """Inputs read once, outputs written once, multiplications and additions of the definition."""
    c, M = case, case["M"]
    if c["kind"] in ("norm", "norm8"):
        each = 2 * _BYTES[c["dtype"]] + 2 * _BYTES[c["residual"]]
        stages = math.log2(c["block"]) + 2 if c["block"] else 0
        return {"bytes": M * c["K"] * each + c["samples"] * c["K"] * _BYTES[c["weight"]],
                "flops": M * c["K"] * (5 + stages)}
    if c["kind"] == "rope":
        n = sum(_axes(c))
        values = M * c["heads"] * (n + c["unrotated"])
        return {"bytes": 2 * values * _BYTES[c["dtype"]] + 12 * c["tokens"] + 4 * n,
                "flops": 3 * M * c["heads"] * n + (4 * values if c["norm"] else 0)}
    half = c["bits"] / 8
    if c["kind"] == "linear":
        out = M * c["N"] * _BYTES[c["dtype"]]
        return {"bytes": 2 * M * c["K"] + half * c["N"] * c["K"] + out * (2 if c["residual"] else 1),
                "flops": 2 * M * c["N"] * c["K"]}
    return {"bytes": M * c["K"] * (2 + 2 * _BYTES[c["dtype"]]) + 2 * half * c["K"] * c["F"],
            "flops": 4 * M * c["K"] * c["F"]}


# ---- the definition in 64 bits --------------------------------------------------------

def _hadamard64(n):
    i = torch.arange(n, device="cuda")
    bits = i.unsqueeze(0) & i.unsqueeze(1)
    odd = torch.zeros_like(bits)
    for j in range(8):
        odd = odd ^ (bits >> j & 1)
    return 1.0 - 2.0 * odd.double()


def _values64(x, block):
    """The values that the 8-bit codes of rows rotated by the Hadamard matrix itself stand for; rows in pieces."""
    out, h = [], _hadamard64(block)
    for v in x.split(max(1, (1 << 26) // x.shape[-1])):
        v = (v.reshape(-1, block) @ h).view_as(v)
        step = v.abs().amax(-1, keepdim=True) / 127.0
        out.append(torch.where(step == 0, v, torch.round(v / step) * step))
    return torch.cat(out)


def _codes64(x, block):
    """The values of the codes as the quantizer's definition fixes them bit for bit: stages, ratio and scale in 32 bits."""
    v = x.float().clone()
    h = 1
    while h < block:
        p = v.view(v.shape[0], -1, 2, h)
        a, b = p[:, :, 0].clone(), p[:, :, 1].clone()
        p[:, :, 0] = a + b
        p[:, :, 1] = a - b
        h *= 2
    top = v.abs().amax(1, keepdim=True).double()
    r = (127.0 / top.clamp(min=1e-300)).float().double()
    return torch.where(top == 0, v.double(), torch.round(v.double() * r) * (top / 127.0).float().double())


def _rows64(w, M):
    w = w.double()
    return w.expand(M, -1) if w.dim() == 1 else w.unsqueeze(1).expand(-1, M // w.shape[0], -1).reshape(M, -1)


def _norm64(x, r, w):
    v = x.double() if r is None else x.double() + r.double()
    n = v * torch.rsqrt(v.pow(2).mean(-1, keepdim=True) + EPS)
    return v, n if w is None else n * _rows64(w, x.shape[0])


def exact(case, seed):
    s = _inputs(case, seed)
    kind, M = case["kind"], case["M"]
    if kind in ("norm", "norm8"):
        v, n = _norm64(s["x"], s["r"], s["w"])
        if kind == "norm8":
            n = _values64(n if s["swap"] is None else n.index_select(1, s["swap"].long()), case["block"])
        return {"y": n} if s["r"] is None else {"y": n, "sum": v}
    if kind == "rope":
        v = s["x"].double()
        if s["w"] is not None:
            v = v * torch.rsqrt(v.pow(2).mean(-1, keepdim=True) + EPS) * s["w"].double()
        n = s["freqs"].numel()
        first, half = 0, []
        for j, d in enumerate(_axes(case)):
            half.append(s["at"][:, j:j + 1].double() * s["freqs"][first:first + d // 2])
            first += d // 2
        turn = torch.cat(half, 1).repeat(M // case["tokens"], 1)
        turn = torch.polar(torch.ones_like(turn), -turn if case["inverse"] else turn).unsqueeze(1)
        if case["interleaved"]:
            z = torch.view_as_real(torch.view_as_complex(v[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * turn).flatten(-2)
        else:
            z = torch.complex(v[..., :n], v[..., n:2 * n]) * turn
            z = torch.cat((z.real, z.imag), -1)
        return torch.cat((z, v[..., 2 * n:]), -1)
    act = {"none": lambda h: h, "gelu": lambda h: h * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (h + 0.044715 * h ** 3)),
           "silu": lambda h: h * torch.sigmoid(h)}
    if kind == "linear":
        y = _codes64(s["x"], case["block"]) @ (s["codes"].double() * s["scale"].double().unsqueeze(1)).t()
        y = act[case["act"]](y if s["b"] is None else y + s["b"].double())
        y = y if s["g"] is None else y * _rows64(s["g"], M)
        return y if s["r"] is None else y + s["r"].double()
    v, n = _norm64(s["x"], s["r"], s["n"])
    h = _values64(n, case["block"]) @ (s["codes1"].double() * s["scale1"].double().unsqueeze(1)).t() + s["b1"].double()
    h = _values64(act["gelu"](h), case["block"]) @ (s["codes2"].double() * s["scale2"].double().unsqueeze(1)).t()
    return v + _rows64(s["g"], M) * (h + s["b2"].double())
