"""Performance cases of the microscaled 4-bit (MX4) operators and of the expert
layer built on them: rotation + MX4 quantizer, MX4 linear and MLP, expert
routing, and the expert MLP.

MX4 is a grid of 4-bit floating-point codes (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6
and their negatives) with one power-of-two scale for 32 consecutive values of
a row: scale 2^e, e = floor(log2(max|x|)) - 2 and at least -126; code = x / 2^e
rounded to the nearest grid value, ties to the even code, at most 6.  `block`
is the size of the Hadamard blocks that rotate a row before it is quantized (0:
no rotation); weights hold the rotation and its 1 / block.

`own = False` computes every operator in elementary torch operations in 32 bits;
`own = True` makes the library's calls.
"""
import math

import torch

own = False

GROUP = 32        # values that share a scale; rows an expert's segment is padded to
_TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}


def _lib():
    import paper_2509_24416_amd as clq
    return clq


def listed():
    return [
        # a few condition tokens through a quantizer: launch and latency only
        dict(name="quantize_few", kind="quantize", M=16, K=1152, block=64, perm=False, dtype="float16"),
        # token count that fills no tile, OBS swap, the largest Hadamard block
        dict(name="quantize_ragged_swap", kind="quantize", M=2777, K=4608, block=128, perm=True, dtype="bfloat16"),
        # the widest input of a video block (fc2's), every token of a step
        dict(name="quantize_video", kind="quantize", M=43200, K=4608, block=64, perm=False, dtype="float16"),
        # one token's qkv linear: the weights are read once for a single row
        dict(name="linear_token", kind="linear", M=1, K=1152, N=3456, block=64, perm=False, bias=True,
             dtype="float16"),
        # sizes that fill no tile, gathered by a swap vector, smallest block
        dict(name="linear_ragged_swap", kind="linear", M=777, K=1216, N=1000, block=32, perm=True, bias=True,
             dtype="bfloat16"),
        # the MLP of a 1024-pixel image transformer's block, 4096 tokens x guidance batch 2
        dict(name="mlp_image", kind="mlp", M=8192, K=1152, F=4608, block=64, act="gelu", dtype="float16"),
        # the widest linear of a video block, every token of a step
        dict(name="linear_video", kind="linear", M=43200, K=1152, N=4608, block=64, perm=False, bias=True,
             dtype="float16"),
        # the router's answer for one token
        dict(name="route_token", kind="route", T=1, E=64, k=6, score="softmax", bias=False, groups=1, top_groups=1,
             renormalize=True),
        # every token of a video step to 8 of 256 experts in 4 of 8 groups, with a balancing bias
        dict(name="route_video", kind="route", T=43200, E=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4,
             renormalize=True),
        # one token under guidance batch 2 through its two experts of 16
        dict(name="experts_few", kind="experts", T=2, K=1152, F=4608, E=16, k=2, block=64, act="gelu", skew=0.5,
             dtype="float16"),
        # an image's tokens through 6 of 64 small gated experts, unevenly loaded
        dict(name="experts_image", kind="experts", T=4096, K=1152, F=768, E=64, k=6, block=64, act="swiglu", skew=1.0,
             dtype="bfloat16"),
        # a video step's tokens through 2 of 16 experts of a whole MLP's width
        dict(name="experts_video", kind="experts", T=43200, K=1152, F=4608, E=16, k=2, block=64, act="gelu", skew=0.5,
             dtype="float16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step):
    return max(1, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step


def draw(rng):
    kind = rng.choices(["quantize", "linear", "mlp", "route", "experts"], [4, 4, 2, 4, 4])[0]
    block = rng.choice([0, 32, 64, 64, 128])
    dtype = rng.choice(["float16", "bfloat16"])
    if kind == "quantize":
        K, M = _width(rng, 64, 12288, max(64, block)), _log_int(rng, 1, 43200)
        while M * K > 43200 * 4608:
            M = M // 2 + 1
        return dict(kind=kind, M=M, K=K, block=block, perm=rng.random() < 0.3, dtype=dtype)
    if kind == "linear":
        K, N, M = _width(rng, 128, 4608, max(64, block)), _log_int(rng, 16, 4608), _log_int(rng, 1, 43200)
        while M * K * N > 43200 * 1152 * 4608 or M * K > 43200 * 2304:
            M = M // 2 + 1
        return dict(kind=kind, M=M, K=K, N=N, block=block, perm=rng.random() < 0.3, bias=rng.random() < 0.8,
                    dtype=dtype)
    if kind == "mlp":
        act = rng.choice(["gelu", "gelu", "swiglu"])
        block = min(block, 64) if act == "swiglu" else block
        K, F, M = _width(rng, 128, 1152, 128), _width(rng, 256, 4608, 128), _log_int(rng, 1, 43200)
        while M * K * F > 43200 * 1152 * 2304:
            M = M // 2 + 1
        return dict(kind=kind, M=M, K=K, F=F, block=block, act=act, dtype=dtype)
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * rng.randint(2, 256 // groups)
        top_groups = rng.randint((groups + 1) // 2, groups)
        k = rng.randint(1, min(8, E // groups * top_groups))
        return dict(kind=kind, T=_log_int(rng, 1, 43200), E=E, k=k, score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, renormalize=rng.random() < 0.7)
    act = rng.choice(["gelu", "swiglu"])
    block = min(block, 64) if act == "swiglu" else block
    K, F, E = _width(rng, 128, 1152, 128), _width(rng, 128, 2304, 128), _log_int(rng, 2, 64)
    k, T = rng.randint(1, min(6, E)), _log_int(rng, 1, 43200)
    while T * k * K * F > 43200 * 1152 * 1152:
        T = T // 2 + 1
    return dict(kind=kind, T=T, K=K, F=F, E=E, k=k, block=block, act=act, skew=rng.choice([0.0, 0.5, 1.0]),
                dtype=dtype)


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


def _weights(g, block, *shape):
    """Rotated weights with 1 / block in them, as a checkpoint holds them: packed codes
    (two a byte, the even column's in the low half) and scale bytes e + 127."""
    w = _normal(g, *shape) / math.sqrt(shape[-1] * max(1, block))
    e = _exponents(w)
    q = _grid(w.unflatten(-1, (-1, GROUP)) * _pow2(-e).unsqueeze(-1)).flatten(-2)
    a = q.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (q < 0).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _swap(g, K):
    return torch.randperm(K, device="cuda", generator=g).to(torch.int32)


def _routing(g, T, E, k, skew):
    """Experts and weights as a router gives them: k of E for each token, some experts
    drawn more often than others."""
    logits = _normal(g, T, E) + skew * _normal(g, E)
    s, ids = torch.sort(torch.softmax(logits, -1), -1, descending=True)
    s, ids = s[:, :k], ids[:, :k].to(torch.int32).contiguous()
    return ids, (s / s.sum(-1, keepdim=True)).contiguous()


def _inputs(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = dict(case)
    if kind in ("quantize", "linear"):
        s["x"] = _activations(g, case["M"], case["K"], case["dtype"])
        s["swap"] = _swap(g, case["K"]) if case["perm"] else None
        if kind == "linear":
            s["w"] = _weights(g, case["block"], case["N"], case["K"])
            s["b"] = (0.1 * _normal(g, case["N"])).to(_TYPES[case["dtype"]]) if case["bias"] else None
    elif kind in ("mlp", "experts"):
        K, F, rows = case["K"], case["F"], case.get("M", case.get("T"))
        lead = (case["E"],) if kind == "experts" else ()
        up = 2 * F if case["act"] == "swiglu" else F
        s["x"] = _activations(g, rows, K, case["dtype"])
        # (the first product brings the outliers' size back to that of a normalised layer)
        c, e = _weights(g, case["block"], *lead, up, K)
        s["w1"] = (c, e - 3)
        s["b1"] = (0.1 * _normal(g, *lead, up)).to(_TYPES[case["dtype"]])
        s["w2"] = _weights(g, case["block"], *lead, K, F)
        s["b2"] = (0.1 * _normal(g, *lead, K)).to(_TYPES[case["dtype"]])
        if kind == "experts":
            s["ids"], s["gates"] = _routing(g, case["T"], case["E"], case["k"], case["skew"])
            # the fullest expert's rows: what the plain form pads every expert to
            s["most"] = int(torch.bincount(s["ids"].flatten(), minlength=case["E"]).max())
    else:
        s["logits"] = 1.5 * _normal(g, case["T"], case["E"])
        s["balance"] = 0.05 * _normal(g, case["E"]) if case["bias"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # weights are laid out once, when a program loads them
        pack = _lib().clq_mx4_pack_weights
        if "w" in s:
            s["qw"] = pack(*s["w"], block=case["block"], perm=s["swap"])
        if "w1" in s:
            s["q1"] = pack(*s["w1"], block=case["block"], gated=case["act"] == "swiglu")
            s["q2"] = pack(*s["w2"], block=case["block"])
    return s


# ---- the plain forms --------------------------------------------------------------

def _pow2(e):
    """2^e for whole e in [-126, 127], from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponents(v):
    """The exponent of each group of 32's scale."""
    m = v.unflatten(-1, (-1, GROUP)).abs().amax(-1)
    return (torch.frexp(m)[1] - 3).clamp(min=-126)


def _grid(v):
    """The nearest e2m1 value, ties to the even code, at most 6 in magnitude."""
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), v)


def _mx4(v):
    """The values that the codes and scales of v stand for."""
    s = _pow2(_exponents(v)).unsqueeze(-1)
    return (_grid(v.unflatten(-1, (-1, GROUP)) / s) * s).flatten(-2)


def _butterflies(v, h, block):
    """Stages h, 2h, ..., block / 2 of the unnormalised Hadamard transform."""
    if h >= block:
        return v
    p = v.unflatten(-1, (-1, 2, h))
    lo, hi = p[..., 0, :], p[..., 1, :]
    return _butterflies(torch.stack((lo + hi, lo - hi), -2).flatten(-3), 2 * h, block)


def _quantized(x, block, swap=None):
    v = x.float()
    v = v if swap is None else v[..., swap.long()]
    return _mx4(_butterflies(v, 1, block))


def _decoded(w):
    """Packed codes and scale bytes as 32-bit values."""
    codes, scales = w
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat((table, -table))
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    return (v.unflatten(-1, (-1, GROUP)) * _pow2(scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


def _activated(h, act):
    if act == "swiglu":   # first half of the channels gates the second
        gate, up = h.chunk(2, -1)
        return gate / (1.0 + torch.exp(-gate)) * up
    return 0.5 * h * (1.0 + torch.tanh(0.7978845608028654 * (h + 0.044715 * h * h * h)))


def _positions(ids, E):
    """Rows of each expert, and the row of each (token, slot) where experts follow one
    another in segments padded to 32 rows and a segment's rows follow the tokens."""
    flat = ids.flatten().long()
    ordered, order = flat.sort(stable=True)
    counts = torch.zeros(E, dtype=torch.int64, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))
    place = torch.arange(flat.numel(), device=ids.device) - (counts.cumsum(0) - counts)[ordered]
    rank = torch.empty_like(flat).index_copy_(0, order, place)
    units = (counts + GROUP - 1) // GROUP
    first = GROUP * (units.cumsum(0) - units)
    return counts.to(torch.int32), (first[flat] + rank).view_as(ids).to(torch.int32), rank.view_as(ids)


def _plain_route(s):
    x, E, k = s["logits"].float(), s["E"], s["k"]
    if s["score"] == "softmax":
        p = torch.exp(x - x.amax(-1, keepdim=True))
        # (the sum in 64 bits: which experts are chosen then hangs on no order of adding)
        score = p / p.double().sum(-1, keepdim=True).float()
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    # (the scores keep the order of the logits; far from 0 they round to one value)
    plain = s["balance"] is None and s["groups"] == 1
    choice = x if plain else score if s["balance"] is None else score + s["balance"]
    if s["groups"] > 1:
        by = choice.unflatten(-1, (s["groups"], -1))
        best = by.sort(-1, descending=True)[0][..., :2].sum(-1)
        kept = best.sort(dim=-1, descending=True, stable=True)[1][:, : s["top_groups"]]
        mask = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        choice = torch.where(mask.unsqueeze(-1), by, -math.inf).flatten(-2)
    ids = choice.sort(dim=-1, descending=True, stable=True)[1][:, :k]
    weights = score.gather(1, ids)
    if s["renormalize"]:
        weights = weights / weights.sum(-1, keepdim=True)
    counts, rows, _ = _positions(ids, E)
    return {"ids": ids.to(torch.int32), "weights": weights, "counts": counts, "rows": rows}


def _plain_experts(s):
    T, k, E, C = s["T"], s["k"], s["E"], s["most"]
    rank = _positions(s["ids"], E)[2]
    place = (s["ids"].long() * C + rank).flatten()
    x = _quantized(s["x"], s["block"])
    rows = torch.zeros(E * C, s["K"], device=x.device).index_copy_(0, place, x.repeat_interleave(k, 0))
    h = torch.bmm(rows.view(E, C, -1), _decoded(s["w1"]).transpose(1, 2).contiguous()) + s["b1"].float().unsqueeze(1)
    h = _quantized(_activated(h, s["act"]), s["block"])
    y = torch.bmm(h, _decoded(s["w2"]).transpose(1, 2).contiguous()) + s["b2"].float().unsqueeze(1)
    y = y.flatten(0, 1)[place].view(T, k, -1)
    return (y * s["gates"].unsqueeze(-1)).sum(1).to(s["x"].dtype)


def _plain(s):
    if s["kind"] == "quantize":
        return _quantized(s["x"], s["block"], s["swap"]).to(torch.bfloat16)
    if s["kind"] == "linear":
        y = _quantized(s["x"], s["block"], s["swap"]) @ _decoded(s["w"]).t()
        return (y if s["b"] is None else y + s["b"].float()).to(s["x"].dtype)
    if s["kind"] == "mlp":
        h = _quantized(s["x"], s["block"]) @ _decoded(s["w1"]).t() + s["b1"].float()
        h = _quantized(_activated(h, s["act"]), s["block"])
        return (h @ _decoded(s["w2"]).t() + s["b2"].float()).to(s["x"].dtype)
    return _plain_route(s) if s["kind"] == "route" else _plain_experts(s)


# ---- one pass -----------------------------------------------------------------------

def run(state):
    s = state
    if not own:
        return _plain(s)
    clq = _lib()
    kind = s["kind"]
    if kind == "route":
        ids, weights = clq.clq_expert_route(s["logits"], s["k"], score=s["score"], bias=s["balance"],
                                            groups=s["groups"], top_groups=s["top_groups"],
                                            renormalize=s["renormalize"])
        plan = clq.clq_expert_plan(ids, s["E"])
        return {"ids": ids, "weights": weights, "counts": plan.counts, "rows": plan.rows}
    if kind == "experts":
        plan = clq.clq_expert_plan(s["ids"], s["E"])
        q = clq.clq_mx4_dispatch(s["x"], plan, block=s["block"])
        h = clq.clq_mx4_experts_mx4(q, plan, s["q1"], s["b1"], act=s["act"], block=s["block"])
        y = clq.clq_mx4_experts(h, plan, s["q2"], s["b2"])
        return clq.clq_expert_combine(y, plan, s["gates"])
    q = clq.clq_mx4_quantize(s["x"], block=s["block"], perm=s.get("swap"))
    if kind == "quantize":
        return clq.clq_mx4_dequantize(q, dtype=torch.bfloat16)
    if kind == "linear":
        return clq.clq_mx4_linear(q, s["qw"], s["b"], dtype=s["x"].dtype)
    h = clq.clq_mx4_linear_mx4(q, s["q1"], s["b1"], act=s["act"], block=s["block"])
    return clq.clq_mx4_linear(h, s["q2"], s["b2"], dtype=s["x"].dtype)


def work(case):
    """Inputs read once, outputs written once, multiplications and additions of the definition.
    Codes are half a byte a value with a scale byte for 32; only experts that a token went to
    are read (their expected number under even routing)."""
    mx = 0.5 + 1.0 / GROUP
    c = case
    stages = math.log2(c["block"]) if c.get("block") else 0
    if c["kind"] == "quantize":
        # read in 16 bits; what is returned are the values, 16 bits each, of the codes
        return {"bytes": c["M"] * c["K"] * (2 + 2), "flops": c["M"] * c["K"] * (stages + 3)}
    if c["kind"] == "linear":
        return {"bytes": 2 * c["M"] * (c["K"] + c["N"]) + mx * c["N"] * c["K"] + 2 * c["N"],
                "flops": 2 * c["M"] * c["N"] * c["K"]}
    if c["kind"] == "route":
        return {"bytes": c["T"] * (4 * c["E"] + 12 * c["k"]) + 4 * c["E"], "flops": 6 * c["T"] * c["E"]}
    up = 2 * c["F"] if c["act"] == "swiglu" else c["F"]
    weights = mx * c["K"] * (up + c["F"]) + 2 * (up + c["K"])
    if c["kind"] == "mlp":
        return {"bytes": 4 * c["M"] * c["K"] + weights, "flops": 2 * c["M"] * c["K"] * (up + c["F"])}
    used = c["E"] * (1.0 - (1.0 - c["k"] / c["E"]) ** c["T"])
    return {"bytes": 4 * c["T"] * c["K"] + 8 * c["T"] * c["k"] + used * weights,
            "flops": 2 * c["T"] * c["k"] * c["K"] * (up + c["F"])}


# ---- the definition in 64 bits --------------------------------------------------------

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _hadamard64(n):
    i = torch.arange(n, device="cuda")
    bits = i.unsqueeze(0) & i.unsqueeze(1)
    odd = torch.zeros_like(bits)
    for j in range(8):
        odd = odd ^ (bits >> j & 1)
    return 1.0 - 2.0 * odd.double()


def _quantized64(x, block, swap=None):
    """Rotates by the Hadamard matrix itself, and picks the grid value by where the midpoints
    of its neighbours lie; rows in pieces."""
    out = []
    for v in x.double().split(max(1, (1 << 26) // x.shape[-1])):
        if swap is not None:
            v = v.index_select(-1, swap.long())
        if block:
            v = (v.reshape(-1, block) @ _hadamard64(block)).view_as(v)
        v = v.reshape(-1, GROUP)
        top = v.abs().amax(1, keepdim=True)
        scale = torch.exp2((torch.floor(torch.log2(top.clamp(min=2.0 ** -124))) - 2.0).clamp(min=-126.0))
        grid = torch.tensor(_GRID, dtype=torch.float64, device="cuda")
        mid = (grid[1:] + grid[:-1]) / 2
        a = (v / scale).abs()
        lower, upper = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)   # they differ on a tie
        pick = torch.where(lower % 2 == 0, lower, upper)
        out.append((torch.copysign(grid[pick], v) * scale).view(-1, x.shape[-1]))
    return torch.cat(out)


def _decoded64(w):
    codes, scales = w
    grid = torch.tensor(_GRID + tuple(-v for v in _GRID), dtype=torch.float64, device="cuda")
    v = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device="cuda")
    v[..., 0::2], v[..., 1::2] = grid[(codes % 16).int()], grid[(codes // 16).int()]
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(GROUP, -1)


def _mlp64(x, w1, b1, w2, b2, act, block):
    h = x @ _decoded64(w1).t() + b1.double()
    if act == "swiglu":
        f = h.shape[-1] // 2
        h = h[:, :f] * torch.sigmoid(h[:, :f]) * h[:, f:]
    else:
        h = h * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (h + 0.044715 * h ** 3))
    return _quantized64(h, block) @ _decoded64(w2).t() + b2.double()


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "route":
        x = s["logits"].double()
        score = torch.softmax(x, -1) if case["score"] == "softmax" else torch.sigmoid(x)
        choice = score if s["balance"] is None else score + s["balance"].double()
        if case["groups"] > 1:
            by = choice.view(case["T"], case["groups"], -1)
            best = by.topk(min(2, by.shape[-1]), -1)[0].sum(-1)
            drop = torch.ones_like(best, dtype=torch.bool)
            drop.scatter_(1, best.topk(case["top_groups"], -1)[1], False)
            choice = by.masked_fill(drop.unsqueeze(-1), -math.inf).reshape(case["T"], -1)
        weights = score.gather(1, choice.topk(case["k"], -1)[1])
        if case["renormalize"]:
            weights = weights / weights.sum(-1, keepdim=True)
        return {"ids": None, "weights": weights, "counts": None, "rows": None}
    x = _quantized64(s["x"], case["block"], s.get("swap"))
    if kind == "quantize":
        return x
    if kind == "linear":
        y = x @ _decoded64(s["w"]).t()
        return y if s["b"] is None else y + s["b"].double()
    if kind == "mlp":
        return _mlp64(x, s["w1"], s["b1"], s["w2"], s["b2"], case["act"], case["block"])
    y = torch.zeros_like(x)
    for e in range(case["E"]):
        token, slot = (s["ids"] == e).nonzero(as_tuple=True)
        if len(token):
            part = _mlp64(x[token], *((s[n][0][e], s[n][1][e]) if n[0] == "w" else s[n][e]
                                      for n in ("w1", "b1", "w2", "b2")), case["act"], case["block"])
            y.index_add_(0, token, part * s["gates"][token, slot].double().unsqueeze(-1))
    return y
