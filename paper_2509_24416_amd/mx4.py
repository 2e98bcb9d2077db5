"""Python binding of the MX4 operators and the expert layer (``include/clq_mx4.h``).

Argument marshalling only, in the manner of the package's other entry points:

    clq_mx4_quantize(X, block=0, perm=None)                    -> MX4
    clq_mx4_quantize_weights(W, block=0, perm=None, gated=False) -> MX4Weight
    clq_mx4_pack_weights(codes, scales, block=0, perm=None, gated=False) -> MX4Weight
    clq_mx4_dequantize(q, dtype=torch.float16)                 -> values
    clq_mx4_linear(q, qw, bias=None)                           -> Y
    clq_mx4_linear_mx4(q, qw, bias=None, act=None, block=0)    -> MX4
    clq_expert_route(logits, top_k, ...)                       -> (ids, weights)
    clq_expert_plan(ids, experts)                              -> ExpertPlan
    clq_mx4_dispatch(X, plan, block=0, perm=None)              -> MX4 in the plan's rows
    clq_mx4_experts(q, plan, qw, bias=None)                    -> Y in the plan's rows
    clq_mx4_experts_mx4(q, plan, qw, bias=None, act=None, block=0) -> MX4 in the plan's rows
    clq_expert_combine(Y, plan, weights)                       -> out

Every call enqueues on the current stream, or on `stream`; what it allocates belongs
to that stream.
"""
import ctypes
from dataclasses import dataclass

import torch

from . import CLQ_ERR_SHAPE, ClqError, _check, _lib, _perm, _ptr, _raw_stream

_i64, _i32, _f32, _p, _sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
_SIGNATURES = {
    "clq_mx4_code_bytes": (_sz, [_i64, _i64, _i32]),
    "clq_mx4_scale_bytes": (_sz, [_i64, _i64, _i32]),
    "clq_mx4_quantize": (_i32, [_p, _i32, _i64, _p, _i64, _i64, _i32, _p, _p, _p]),
    "clq_mx4_quantize_weights": (_i32, [_p, _i32, _p, _i64, _i64, _i64, _i32, _i32, _p, _p, _p]),
    "clq_mx4_pack_weights": (_i32, [_p, _p, _i64, _i64, _i64, _i32, _p, _p, _p]),
    "clq_mx4_dequantize": (_i32, [_p, _p, _i32, _i32, _i64, _i64, _i64, _i32, _p, _i64, _p]),
    "clq_mx4_linear": (_i32, [_p, _p, _p, _p, _p, _i32, _i64, _i64, _i64, _i32, _p, _i64, _p]),
    "clq_mx4_linear_mx4": (_i32, [_p, _p, _p, _p, _p, _i32, _i64, _i64, _i64, _i32, _i32, _p, _p, _p]),
    "clq_expert_route": (_i32, [_p, _i32, _i64, _i64, _i64, _i32, _i32, _p, _i32, _i32, _i32, _f32, _p, _p, _p]),
    "clq_expert_plan_rows": (_i64, [_i64, _i64, _i64]),
    "clq_expert_plan_ints": (_i64, [_i64]),
    "clq_expert_plan_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "clq_expert_plan": (_i32, [_p, _i64, _i64, _i64, _p, _p, _p, _p, _sz, _p]),
    "clq_mx4_dispatch": (_i32, [_p, _i32, _i64, _p, _i64, _i64, _i64, _i64, _i32, _p, _p, _p, _p, _p]),
    "clq_mx4_experts": (_i32, [_p, _p, _p, _i64, _i64, _i64, _p, _p, _p, _i32, _i64, _i64, _i32, _p, _i64, _p]),
    "clq_mx4_experts_mx4": (_i32, [_p, _p, _p, _i64, _i64, _i64, _p, _p, _p, _i32, _i64, _i64, _i32, _i32, _p, _p,
                                   _p]),
    "clq_expert_combine": (_i32, [_p, _i32, _i64, _p, _p, _i64, _i64, _i64, _i64, _p, _i32, _i64, _p]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

MX4_EXPORTS = tuple(_SIGNATURES)
__all__ = ["MX4", "MX4Weight", "ExpertPlan", "MX4_EXPORTS", *MX4_EXPORTS]

_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_ACTS = {None: 0, "none": 0, "gelu": 1, "swiglu": 2}
_SCORES = {"softmax": 0, "sigmoid": 1}


class MX4:
    """Activations quantized to MX4: `rows` rows of `K` values, rotated by blocks of `block`.
    One uint8 buffer holds the codes, then the scales (opaque layouts)."""
    __slots__ = ("data", "rows", "K", "block")

    def __init__(self, data, rows, K, block=0):
        self.data, self.rows, self.K, self.block = data, rows, K, block
        if data.is_cuda:
            _bytes(data, _code_bytes(rows, K) + _scale_bytes(rows, K), "data")

    @property
    def codes(self):
        return self.data[:_code_bytes(self.rows, self.K)]

    @property
    def scales(self):
        c = _code_bytes(self.rows, self.K)
        return self.data[c:c + _scale_bytes(self.rows, self.K)]

    def __repr__(self):
        return f"MX4(rows={self.rows}, K={self.K}, block={self.block})"


@dataclass(slots=True)
class MX4Weight:
    """An N x K weight matrix in MX4, or `experts` of them."""
    codes: torch.Tensor     # uint8, opaque layout, expert after expert
    scales: torch.Tensor    # uint8
    N: int
    K: int
    block: int = 0
    perm: torch.Tensor = None
    experts: int = None     # None: a plain matrix
    gated: bool = False

    def __post_init__(self):
        if self.codes.is_cuda:
            rows = _weight_rows(self.experts, self.N)
            _bytes(self.codes, _code_bytes(rows, self.K), "codes")
            _bytes(self.scales, _scale_bytes(rows, self.K), "scales")
            _together(self.codes.device, "scales", self.scales)


class ExpertPlan:
    """Assignments sorted by expert: `tokens` x `top_k` of them to `experts` experts, in buffers
    of `plan_rows` rows.  One int32 buffer holds the tables, the rows and the sources."""
    __slots__ = ("data", "tokens", "top_k", "experts", "plan_rows", "at_rows", "at_source", "dispatched")

    def __init__(self, data, tokens, top_k, experts, plan_rows, ints):
        self.data, self.tokens, self.top_k, self.experts, self.plan_rows = data, tokens, top_k, experts, plan_rows
        self.at_rows, self.at_source, self.dispatched = ints, ints + tokens * top_k, set()

    @property
    def dtype(self):
        """The type of the tokens dispatched with this plan; None before, and where there were two."""
        return next(iter(self.dispatched)) if len(self.dispatched) == 1 else None

    @property
    def counts(self):
        """int32 [experts]: assignments of each expert."""
        return self.data[:self.experts]

    @property
    def rows(self):
        """int32 [tokens, top_k]: the row of each assignment, -1 for none."""
        return self.data[self.at_rows:self.at_source].view(self.tokens, self.top_k)

    @property
    def source(self):
        """int32 [plan_rows]: the token of each row in use, -1 on padding."""
        return self.data[self.at_source:]

    def offsets(self):
        """int32 [experts + 1]: each expert's first row, a multiple of 32, and the end of the last
        one's."""
        return 32 * self.data[self.experts:2 * self.experts + 1]


def _dev(t, name, dtypes):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    return t


_HALF = (torch.float16, torch.bfloat16)


def _together(device, name, t):
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


def _rows2d(X, name, dtypes=_HALF):
    """Rows, columns, row stride of a matrix."""
    _dev(X, name, dtypes)
    if X.dim() != 2:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    M, K = X.shape
    ld, step = X.stride()
    if step != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    # (a single row has no stride of its own; torch gives such a view any)
    return M, K, ld if M > 1 else (K + 7) & ~7


def _gather(perm, K, device):
    _together(device, "perm", _perm(perm, K))
    return perm.data_ptr()


# Every call runs on the current stream of its tensors' device.  One given a stream, or
# tensors of another device, calls itself again with that made current, so that what it
# allocates belongs there too.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _elsewhere(device, stream):
    if stream is None:
        return torch.cuda.device(device)
    _together(device, "stream", stream)
    return torch.cuda.stream(stream)


def _bytes(t, n, name):
    if t.dtype is not torch.uint8 or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous uint8 tensor of at least {n} bytes")


def _weight_rows(experts, N):
    return (experts or 1) * ((N + 63) // 64 * 64)


def _code_bytes(rows, K):
    return (rows + 31) // 32 * 32 * (K // 2)


def _scale_bytes(rows, K):
    return (rows + 31) // 32 * ((K + 255) // 256) * 256


def clq_mx4_code_bytes(rows, K, weights=False):
    return _lib.clq_mx4_code_bytes(rows, K, int(weights))


def clq_mx4_scale_bytes(rows, K, weights=False):
    return _lib.clq_mx4_scale_bytes(rows, K, int(weights))


def _buffer(out, rows, K, block, device, where):
    """A buffer for an MX4 of that shape, the caller's, checked, or a new one; its codes' and
    scales' pointers."""
    if not 0 < rows < 2147483648 or not 64 <= K <= 32768 or K & 63:
        raise ClqError(CLQ_ERR_SHAPE, where)
    units = (rows + 31) >> 5
    codes = units * K << 4
    n = codes + (units * ((K + 255) >> 8) << 8)
    if out is None:
        data = torch.empty(n, dtype=torch.uint8, device=device)
        out = object.__new__(MX4)   # (of that size: nothing to check)
        out.data = data
    else:
        data = _dev(out.data, "out", (torch.uint8,))
        if data.numel() < n or not data.is_contiguous():
            raise ValueError("the output's buffer is too small")
        _together(device, "out", data)
    p = data.data_ptr()
    return out, p, p + codes


def _holds(out, rows, K, block):
    """`out` once a call has filled it (one that was refused leaves it what it was)."""
    out.rows, out.K, out.block = rows, K, block
    return out


# What a call reads and writes, as (address, pieces, bytes between them, bytes of each).
def _meet(a, b):
    """Whether two of those overlap (two sets of pieces at different distances: not looked at)."""
    (at, n, pitch, width), (at2, n2, pitch2, width2) = ((x[0], 1, 1, x[1] * x[3]) if x[1] == 1 or x[2] == x[3] else x
                                                     for x in (a, b))
    pitch, pitch2 = (pitch2 if n == 1 else pitch), (pitch if n2 == 1 else pitch2)
    if pitch != pitch2:
        return False
    # the first piece i of a, counted from piece 0 of b, that ends behind b's start
    i = max((at2 - at - width) // max(pitch, 1) + 1, 1 - n2)
    return i < n and i * pitch < at2 - at + width2


def _mx4_bytes(data, rows, K):
    n = _code_bytes(rows, K) + _scale_bytes(rows, K)
    return data.data_ptr(), 1, n, n


def _row_bytes(t, rows, columns, ld):
    size = t.element_size()
    return t.data_ptr(), rows, ld * size, columns * size


def _weight_bytes(qw):
    rows = _weight_rows(qw.experts, qw.N)
    sizes = _code_bytes(rows, qw.K), _scale_bytes(rows, qw.K)
    return tuple((t.data_ptr(), 1, n, n) for t, n in zip((qw.codes, qw.scales), sizes))


def _apart(out, *inputs):
    """An output of the caller's must not lie in what the launch reads."""
    if any(_meet(out, x) for x in inputs):
        raise ValueError("the output overlaps an input")


def clq_mx4_quantize(X, block=0, perm=None, out=None, stream=None):
    """Rotates each row by blocks of `block` (0: none), after gathering its columns by
    `perm`, and quantizes it to MX4.  X: fp16 or bf16 [M, K], any row stride that is a
    multiple of 8.  out: an MX4 whose buffer is reused."""
    M, K, ldx = _rows2d(X, "X")
    device = X.device
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_quantize(X, block, perm, out)
    if out is not None:
        _apart(_mx4_bytes(out.data, M, K), _row_bytes(X, M, K, ldx))
    q, codes, scales = _buffer(out, M, K, block, device, "clq_mx4_quantize")
    _check(_lib.clq_mx4_quantize(X.data_ptr(), _TYPES[X.dtype], ldx, None if perm is None else _gather(perm, K, device),
                                 M, K, block, codes, scales, _raw_stream(i)), "clq_mx4_quantize")
    return _holds(q, M, K, block)


def _weight_shape(W, name):
    if W.dim() not in (2, 3) or not W.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [N, K] or [experts, N, K] tensor")
    return (None, *W.shape) if W.dim() == 2 else tuple(W.shape)


def _weight(experts, N, K, block, perm, gated, device, where):
    cb, sb = _lib.clq_mx4_code_bytes(N, K, 1), _lib.clq_mx4_scale_bytes(N, K, 1)
    if cb == 0:
        raise ClqError(CLQ_ERR_SHAPE, where)
    e = experts or 1
    return MX4Weight(torch.empty(e * cb, dtype=torch.uint8, device=device),
                     torch.empty(e * sb, dtype=torch.uint8, device=device), N, K, block, perm, experts, gated)


def clq_mx4_quantize_weights(W, block=0, perm=None, gated=False, stream=None):
    """Rotates and quantizes weights, fp16 or bf16 [N, K] or [experts, N, K]; the rotation's
    1 / block is in them.  gated: the first N / 2 rows are the gates of the others (for
    act="swiglu")."""
    _dev(W, "W", _HALF)
    experts, N, K = _weight_shape(W, "W")
    device = W.device
    if stream is not None or _current_device() != device.index:
        with _elsewhere(device, stream):
            return clq_mx4_quantize_weights(W, block, perm, gated)
    p = None if perm is None else _gather(perm, K, device)
    qw = _weight(experts, N, K, block, perm, gated, device, "clq_mx4_quantize_weights")
    _check(_lib.clq_mx4_quantize_weights(W.data_ptr(), _TYPES[W.dtype], p, experts or 1, N, K, block, int(gated),
                                         qw.codes.data_ptr(), qw.scales.data_ptr(), _raw_stream(device.index)),
           "clq_mx4_quantize_weights")
    return qw


def clq_mx4_pack_weights(codes, scales, block=0, perm=None, gated=False, stream=None):
    """Lays out weights that are MX4 already: uint8 codes [..., N, K / 2] (the even column in the
    low half) and scale bytes [..., N, K / 32].  block, perm: the rotation they hold."""
    _dev(codes, "codes", (torch.uint8,))
    _dev(scales, "scales", (torch.uint8,))
    experts, N, half = _weight_shape(codes, "codes")
    K, device = 2 * half, codes.device
    if scales.shape != (*codes.shape[:-1], K // 32) or not scales.is_contiguous():
        raise ValueError("scales must be contiguous, one byte for 32 codes of each row")
    _together(device, "scales", scales)
    if perm is not None:
        _gather(perm, K, device)
    if stream is not None or _current_device() != device.index:
        with _elsewhere(device, stream):
            return clq_mx4_pack_weights(codes, scales, block, perm, gated)
    qw = _weight(experts, N, K, block, perm, gated, device, "clq_mx4_pack_weights")
    _check(_lib.clq_mx4_pack_weights(codes.data_ptr(), scales.data_ptr(), experts or 1, N, K, int(gated),
                                     qw.codes.data_ptr(), qw.scales.data_ptr(), _raw_stream(device.index)),
           "clq_mx4_pack_weights")
    return qw


def clq_mx4_dequantize(q, dtype=torch.float16, out=None, stream=None):
    """The values that an MX4 or MX4Weight stands for (still rotated): [rows, K], [N, K] or
    [experts, N, K] of fp16, bf16 or fp32."""
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be fp16, bf16 or fp32, got {dtype}")
    K = q.K
    if isinstance(q, MX4Weight):
        w, gated, rows, mats = 1, int(q.gated), q.N, q.experts or 1
        shape = (mats, rows, K) if q.experts else (rows, K)
        device, c, s = q.codes.device, q.codes.data_ptr(), q.scales.data_ptr()
    else:
        w, gated, rows, mats, shape, device = 0, 0, q.rows, 1, (q.rows, K), q.data.device
        c = q.data.data_ptr()
        s = c + _code_bytes(rows, K)
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_dequantize(q, dtype, out)
    if out is None:
        out = torch.empty(*shape, dtype=dtype, device=device)
    else:
        if _dev(out, "out", (dtype,)).shape != shape or not out.is_contiguous():
            raise ValueError(f"out must be a contiguous {shape} tensor")
        _together(device, "out", out)
        _apart(_row_bytes(out, out.numel() // K, K, K), *(_weight_bytes(q) if w else (_mx4_bytes(q.data, rows, K),)))
    _check(_lib.clq_mx4_dequantize(c, s, w, gated, mats, rows, K, _TYPES[dtype], out.data_ptr(), K, _raw_stream(i)),
           "clq_mx4_dequantize")
    return out


def _product(q, qw, bias, experts):
    """Checks the operands of a product; their device, and the bias's pointer and type."""
    if not isinstance(q, MX4) or not isinstance(qw, MX4Weight):
        raise TypeError("the operands must be an MX4 and an MX4Weight")
    if q.K != qw.K:
        raise ValueError(f"inputs have {q.K} columns, weights {qw.K}")
    if q.block != qw.block:
        raise ValueError(f"inputs are rotated by blocks of {q.block}, weights by {qw.block}")
    if qw.experts != experts:
        raise ValueError(f"weights hold {qw.experts} experts, not {experts}")
    device = q.data.device
    _together(device, "weights", qw.codes)
    if bias is None:
        return device, None, 0
    _dev(bias, "bias", _HALF)
    if bias.shape != ((qw.N,) if experts is None else (experts, qw.N)) or not bias.is_contiguous():
        raise ValueError("bias must be a contiguous [N] or [experts, N] tensor")
    _together(device, "bias", bias)
    return device, bias.data_ptr(), _TYPES[bias.dtype]


def _output(out, rows, N, dtype, device):
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be fp16, bf16 or fp32, got {dtype}")
    if out is None:   # rows on 16-byte boundaries
        ld = (N + 7) // 8 * 8
        out = torch.empty(rows, ld, dtype=dtype, device=device)
        return (out if ld == N else out[:, :N]), ld
    r, n, ld = _rows2d(out, "out", (dtype,))
    if r < rows or n != N:
        raise ValueError(f"out must be [{rows}, {N}]")
    _together(device, "out", out)
    return out, ld


def _act(act):
    if act not in _ACTS:
        raise ValueError(f"act must be None, 'gelu' or 'swiglu', not {act!r}")
    return _ACTS[act]


def _columns(qw, act):
    if (act == 2) != bool(qw.gated):
        raise ValueError("act='swiglu' takes gated weights, every other activation plain ones")
    return qw.N // 2 if act == 2 else qw.N


def clq_mx4_linear(q, qw, bias=None, dtype=torch.float16, out=None, stream=None):
    """Y = X . W^T + bias, fp16, bf16 or fp32 [M, N]."""
    device, b, bt = _product(q, qw, bias, None)
    if qw.gated:
        raise ValueError("gated weights go with clq_mx4_linear_mx4(act='swiglu')")
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_linear(q, qw, bias, dtype, out)
    M, K, N = q.rows, q.K, qw.N
    Y, ld = _output(out, M, N, dtype, device)
    if out is not None:
        _apart(_row_bytes(Y, M, N, ld), _mx4_bytes(q.data, M, K), *_weight_bytes(qw))
    p = q.data.data_ptr()
    _check(_lib.clq_mx4_linear(p, p + _code_bytes(M, K), qw.codes.data_ptr(), qw.scales.data_ptr(), b, bt, M, N, K,
                               _TYPES[dtype], Y.data_ptr(), ld, _raw_stream(i)), "clq_mx4_linear")
    return Y


def clq_mx4_linear_mx4(q, qw, bias=None, act=None, block=0, out=None, stream=None):
    """act(X . W^T + bias), rotated by blocks of `block` and quantized to MX4 without leaving
    fp32 in between: the input of the next product.  act: None, "gelu" (tanh form) or "swiglu"
    (gated weights, N / 2 columns)."""
    a = _act(act)
    device, b, bt = _product(q, qw, bias, None)
    if out is not None:
        _apart(_mx4_bytes(out.data, q.rows, _columns(qw, a)), _mx4_bytes(q.data, q.rows, q.K), *_weight_bytes(qw))
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_linear_mx4(q, qw, bias, act, block, out)
    M, K, C = q.rows, q.K, _columns(qw, a)
    o, codes, scales = _buffer(out, M, C, block, device, "clq_mx4_linear_mx4")
    p = q.data.data_ptr()
    _check(_lib.clq_mx4_linear_mx4(p, p + _code_bytes(M, K), qw.codes.data_ptr(), qw.scales.data_ptr(), b, bt, M, qw.N,
                                   K, a, block, codes, scales, _raw_stream(i)), "clq_mx4_linear_mx4")
    return _holds(o, M, C, block)


def clq_expert_route(logits, top_k, score="softmax", bias=None, groups=1, top_groups=1, renormalize=True, scale=1.0,
                     stream=None):
    """The top_k experts of each token and their weights: (ids int32 [T, top_k], weights fp32).
    logits: fp32, fp16 or bf16 [T, experts].  score: "softmax" or "sigmoid".  bias: fp32
    [experts], added for the ranking alone.  groups, top_groups: only the experts of the best
    top_groups of `groups` groups take part.  scale multiplies the weights."""
    _dev(logits, "logits", _TYPES)
    if logits.dim() != 2:
        raise ValueError("logits must be 2-D with unit column stride")
    (T, E), (ld, step) = logits.shape, logits.stride()
    if step != 1 and E != 1:
        raise ValueError("logits must be 2-D with unit column stride")
    if score not in _SCORES:
        raise ValueError(f"score must be 'softmax' or 'sigmoid', not {score!r}")
    device = logits.device
    i = device.index
    b = None
    if bias is not None:
        _dev(bias, "bias", (torch.float32,))
        if bias.shape != (E,) or not bias.is_contiguous():
            raise ValueError(f"bias must be a contiguous fp32 [{E}] tensor")
        _together(device, "bias", bias)
        b = bias.data_ptr()
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_expert_route(logits, top_k, score, bias, groups, top_groups, renormalize, scale)
    ids = torch.empty(T, top_k, dtype=torch.int32, device=device)
    weights = torch.empty(T, top_k, dtype=torch.float32, device=device)
    # (a single row has no stride of its own)
    _check(_lib.clq_expert_route(logits.data_ptr(), _TYPES[logits.dtype], ld if T > 1 else E, T, E, top_k,
                                 _SCORES[score], b, groups, top_groups, int(renormalize), scale, ids.data_ptr(),
                                 weights.data_ptr(), _raw_stream(i)), "clq_expert_route")
    return ids, weights


def clq_expert_plan_rows(tokens, top_k, experts):
    return _lib.clq_expert_plan_rows(tokens, top_k, experts)


def clq_expert_plan_ints(experts):
    return _lib.clq_expert_plan_ints(experts)


def clq_expert_plan_workspace_bytes(tokens, top_k, experts):
    return _lib.clq_expert_plan_workspace_bytes(tokens, top_k, experts)


def clq_expert_plan(ids, experts, stream=None):
    """Sorts the assignments ids (int32 [T, top_k]; entries outside 0 .. experts - 1 get no
    row) by expert."""
    _dev(ids, "ids", (torch.int32,))
    if ids.dim() != 2 or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous int32 [tokens, top_k] tensor")
    T, k = ids.shape
    device = ids.device
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_expert_plan(ids, experts)
    n = _lib.clq_expert_plan_rows(T, k, experts)
    if n == 0:
        raise ClqError(CLQ_ERR_SHAPE, "clq_expert_plan")
    nt, nw = _lib.clq_expert_plan_ints(experts), _lib.clq_expert_plan_workspace_bytes(T, k, experts)
    data = torch.empty(nt + T * k + n, dtype=torch.int32, device=device)
    ws = torch.empty(nw, dtype=torch.uint8, device=device) if nw else None
    p = data.data_ptr()
    _check(_lib.clq_expert_plan(ids.data_ptr(), T, k, experts, p, p + 4 * nt, p + 4 * (nt + T * k), _ptr(ws), nw,
                                _raw_stream(i)), "clq_expert_plan")
    return ExpertPlan(data, T, k, experts, n, nt)


def clq_mx4_dispatch(X, plan, block=0, perm=None, out=None, stream=None):
    """clq_mx4_quantize of the tokens X [T, K] into the plan's rows, expert after expert."""
    T, K, ldx = _rows2d(X, "X")
    if T != plan.tokens:
        raise ValueError(f"X has {T} tokens, the plan {plan.tokens}")
    device = X.device
    i = device.index
    _together(device, "plan", plan.data)
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_dispatch(X, plan, block, perm, out)
    g = None if perm is None else _gather(perm, K, device)
    n = plan.plan_rows
    if out is not None:
        _apart(_mx4_bytes(out.data, n, K), _row_bytes(X, T, K, ldx))
    q, codes, scales = _buffer(out, n, K, block, device, "clq_mx4_dispatch")
    t = plan.data.data_ptr()
    _check(_lib.clq_mx4_dispatch(X.data_ptr(), _TYPES[X.dtype], ldx, g, T, plan.top_k, plan.experts, K, block, t,
                                 t + 4 * plan.at_source, codes, scales, _raw_stream(i)), "clq_mx4_dispatch")
    plan.dispatched.add(X.dtype)
    return _holds(q, n, K, block)


def _plan_operands(q, plan, qw, bias):
    r = _product(q, qw, bias, plan.experts)
    if q.rows != plan.plan_rows:
        raise ValueError(f"inputs have {q.rows} rows, the plan {plan.plan_rows}")
    _together(r[0], "plan", plan.data)
    return r


def clq_mx4_experts(q, plan, qw, bias=None, dtype=None, out=None, stream=None):
    """Each row of the plan times its expert's weights: Y [plan.plan_rows, N] of fp16, bf16 or fp32;
    rows past the last expert's are left as they were.  dtype: by default that of `out`, or fp32,
    so that a sum of results is rounded once."""
    device, b, bt = _plan_operands(q, plan, qw, bias)
    if qw.gated:
        raise ValueError("gated weights go with clq_mx4_experts_mx4(act='swiglu')")
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_experts(q, plan, qw, bias, dtype, out)
    M, K, N = q.rows, q.K, qw.N
    # (16-bit results make 1.4 times the error of one rounding in the sum, and halve the bytes; whole
    # layers, us, 16 bits / fp32: 512 tokens to 2 of 16 experts of width 1152 46 / 48, 4096 102 / 115,
    # 43200 716 / 842; 4096 to 6 of 64 105 / 136)
    if dtype is None:
        dtype = torch.float32 if out is None else out.dtype
    Y, ld = _output(out, M, N, dtype, device)
    if out is not None:
        _apart(_row_bytes(Y, M, N, ld), _mx4_bytes(q.data, M, K), *_weight_bytes(qw))
    p = q.data.data_ptr()
    _check(_lib.clq_mx4_experts(p, p + _code_bytes(M, K), plan.data.data_ptr(), plan.tokens, plan.top_k, plan.experts,
                                qw.codes.data_ptr(), qw.scales.data_ptr(), b, bt, N, K, _TYPES[dtype], Y.data_ptr(),
                                ld, _raw_stream(i)), "clq_mx4_experts")
    return Y


def clq_mx4_experts_mx4(q, plan, qw, bias=None, act=None, block=0, out=None, stream=None):
    """clq_mx4_linear_mx4 with each row times its expert's weights."""
    a = _act(act)
    device, b, bt = _plan_operands(q, plan, qw, bias)
    if out is not None:
        _apart(_mx4_bytes(out.data, q.rows, _columns(qw, a)), _mx4_bytes(q.data, q.rows, q.K), *_weight_bytes(qw))
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_mx4_experts_mx4(q, plan, qw, bias, act, block, out)
    M, K, C = q.rows, q.K, _columns(qw, a)
    o, codes, scales = _buffer(out, M, C, block, device, "clq_mx4_experts_mx4")
    p = q.data.data_ptr()
    _check(_lib.clq_mx4_experts_mx4(p, p + _code_bytes(M, K), plan.data.data_ptr(), plan.tokens, plan.top_k,
                                    plan.experts, qw.codes.data_ptr(), qw.scales.data_ptr(), b, bt, qw.N, K, a, block,
                                    codes, scales, _raw_stream(i)), "clq_mx4_experts_mx4")
    return _holds(o, M, C, block)


def clq_expert_combine(Y, plan, weights, dtype=None, out=None, stream=None):
    """out[t] = sum over the slots of weights[t, j] * Y[plan.rows[t, j]], in fp32.  dtype: by default
    that of `out`, or of the tokens dispatched with the plan (none: Y's; to be named if there were
    tokens of two types)."""
    r, N, ldy = _rows2d(Y, "Y", _TYPES)
    _dev(weights, "weights", (torch.float32,))
    T, k = plan.tokens, plan.top_k
    if r < plan.plan_rows or weights.shape != (T, k) or not weights.is_contiguous():
        raise ValueError("Y and weights must have the plan's rows and slots")
    device = Y.device
    i = device.index
    _together(device, "weights", weights)
    _together(device, "plan", plan.data)
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_expert_combine(Y, plan, weights, dtype, out)
    if dtype is None and out is None and len(plan.dispatched) > 1:
        raise ValueError("tokens of two types were dispatched with the plan: name the result's dtype")
    if dtype is None:
        dtype = out.dtype if out is not None else plan.dtype or Y.dtype
    o, ld = _output(out, T, N, dtype, device)
    if out is not None:
        _apart(_row_bytes(o, T, N, ld), _row_bytes(Y, plan.plan_rows, N, ldy))
    _check(_lib.clq_expert_combine(Y.data_ptr(), _TYPES[Y.dtype], ldy, plan.data.data_ptr() + 4 * plan.at_rows,
                                   weights.data_ptr(), T, k, plan.experts, N, o.data_ptr(), _TYPES[dtype], ld,
                                   _raw_stream(i)), "clq_expert_combine")
    return o
