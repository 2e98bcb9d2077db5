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
    "clq_expert_combine": (_i32, [_p, _i32, _i64, _p, _p, _i64, _i64, _i64, _i64, _p, _i64, _p]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

MX4_EXPORTS = tuple(_SIGNATURES)
__all__ = ["MX4", "MX4Weight", "ExpertPlan", "MX4_EXPORTS", *MX4_EXPORTS]

_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_ACTS = {None: 0, "none": 0, "gelu": 1, "swiglu": 2}
_SCORES = {"softmax": 0, "sigmoid": 1}


@dataclass(slots=True)
class MX4:
    """Activations quantized to MX4: `rows` rows of `K` values (opaque layouts)."""
    codes: torch.Tensor     # uint8
    scales: torch.Tensor    # uint8
    rows: int
    K: int
    block: int = 0


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


@dataclass(slots=True)
class ExpertPlan:
    """Assignments sorted by expert.  Expert e's rows start at offsets()[e], a multiple of 32."""
    tokens: int
    top_k: int
    experts: int
    plan_rows: int          # rows that buffers of a plan of this size have
    tables: torch.Tensor    # int32
    rows: torch.Tensor      # int32 [tokens, top_k], -1: no row
    source: torch.Tensor    # int32 [plan_rows], the rows' tokens

    @property
    def counts(self):
        """int32 [experts]: assignments of each expert."""
        return self.tables[:self.experts]

    def offsets(self):
        """int32 [experts + 1]: each expert's first row, and the end of the last one's."""
        return 32 * self.tables[self.experts:2 * self.experts + 1]


def _dev(t, name, dtypes):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    return t


_HALF = (torch.float16, torch.bfloat16)


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")


def _rows2d(X, name, dtypes=_HALF):
    _dev(X, name, dtypes)
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    # (a single row has no stride of its own; torch gives such a view any)
    return X.shape[0], X.shape[1], X.stride(0) if X.shape[0] > 1 else max(X.stride(0), -(-X.shape[1] // 8) * 8)


class _On:
    """The raw stream of a call; allocations inside belong to it."""
    __slots__ = ("guard", "device", "given")

    def __init__(self, device, stream):
        self.device, self.given = device, stream
        self.guard = None

    def __enter__(self):
        if self.given is None:
            if torch.cuda.current_device() != self.device.index:
                self.guard = torch.cuda.device(self.device)
                self.guard.__enter__()
            return _raw_stream(self.device.index)
        self.guard = torch.cuda.stream(self.given)
        self.guard.__enter__()
        return self.given.cuda_stream

    def __exit__(self, *e):
        if self.guard is not None:
            self.guard.__exit__(*e)


def clq_mx4_code_bytes(rows, K, weights=False):
    return _lib.clq_mx4_code_bytes(rows, K, int(weights))


def clq_mx4_scale_bytes(rows, K, weights=False):
    return _lib.clq_mx4_scale_bytes(rows, K, int(weights))


def _buffers(out, rows, K, device, where, block=0):
    """An MX4 of that shape: the caller's, checked, or a new one."""
    cb, sb = _lib.clq_mx4_code_bytes(rows, K, 0), _lib.clq_mx4_scale_bytes(rows, K, 0)
    if cb == 0:
        raise ClqError(CLQ_ERR_SHAPE, where)
    if out is None:
        return MX4(torch.empty(cb, dtype=torch.uint8, device=device),
                   torch.empty(sb, dtype=torch.uint8, device=device), rows, K, block)
    for t, n in ((out.codes, cb), (out.scales, sb)):
        if _dev(t, "out", (torch.uint8,)).numel() < n or not t.is_contiguous():
            raise ValueError("the output's buffers are too small")
    _same_device(device, out=out.codes)
    out.rows, out.K, out.block = rows, K, block
    return out


def clq_mx4_quantize(X, block=0, perm=None, out=None, stream=None):
    """Rotates each row by blocks of `block` (0: none), after gathering its columns by
    `perm`, and quantizes it to MX4.  X: fp16 or bf16 [M, K], any row stride that is a
    multiple of 8.  out: an MX4 whose buffers are reused."""
    M, K, ldx = _rows2d(X, "X")
    perm = _perm(perm, K)
    _same_device(X.device, perm=perm)
    with _On(X.device, stream) as s:
        q = _buffers(out, M, K, X.device, "clq_mx4_quantize", block)
        _check(_lib.clq_mx4_quantize(X.data_ptr(), _TYPES[X.dtype], ldx, _ptr(perm), M, K, block,
                                     q.codes.data_ptr(), q.scales.data_ptr(), s), "clq_mx4_quantize")
    return q


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
    perm = _perm(perm, K)
    _same_device(W.device, perm=perm)
    with _On(W.device, stream) as s:
        qw = _weight(experts, N, K, block, perm, gated, W.device, "clq_mx4_quantize_weights")
        _check(_lib.clq_mx4_quantize_weights(W.data_ptr(), _TYPES[W.dtype], _ptr(perm), experts or 1, N, K, block,
                                             int(gated), qw.codes.data_ptr(), qw.scales.data_ptr(), s),
               "clq_mx4_quantize_weights")
    return qw


def clq_mx4_pack_weights(codes, scales, block=0, perm=None, gated=False, stream=None):
    """Lays out weights that are MX4 already: uint8 codes [..., N, K / 2] (the even column in the
    low half) and scale bytes [..., N, K / 32].  block, perm: the rotation they hold."""
    _dev(codes, "codes", (torch.uint8,))
    _dev(scales, "scales", (torch.uint8,))
    experts, N, half = _weight_shape(codes, "codes")
    K = 2 * half
    perm = _perm(perm, K)
    if scales.shape != (*codes.shape[:-1], K // 32) or not scales.is_contiguous():
        raise ValueError("scales must be contiguous, one byte for 32 codes of each row")
    _same_device(codes.device, scales=scales, perm=perm)
    with _On(codes.device, stream) as s:
        qw = _weight(experts, N, K, block, perm, gated, codes.device, "clq_mx4_pack_weights")
        _check(_lib.clq_mx4_pack_weights(codes.data_ptr(), scales.data_ptr(), experts or 1, N, K, int(gated),
                                         qw.codes.data_ptr(), qw.scales.data_ptr(), s), "clq_mx4_pack_weights")
    return qw


def clq_mx4_dequantize(q, dtype=torch.float16, out=None, stream=None):
    """The values that an MX4 or MX4Weight stands for (still rotated): [rows, K], [N, K] or
    [experts, N, K] of fp16, bf16 or fp32."""
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be fp16, bf16 or fp32, got {dtype}")
    w = isinstance(q, MX4Weight)
    rows = q.N if w else q.rows
    mats = (q.experts or 1) if w else 1
    shape = (mats, rows, q.K) if w and q.experts else (rows, q.K)
    with _On(q.codes.device, stream) as s:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=q.codes.device)
        elif _dev(out, "out", (dtype,)).shape != shape or not out.is_contiguous():
            raise ValueError(f"out must be a contiguous {shape} tensor")
        _same_device(q.codes.device, out=out)
        _check(_lib.clq_mx4_dequantize(q.codes.data_ptr(), q.scales.data_ptr(), int(w), int(w and q.gated), mats, rows,
                                       q.K, _TYPES[dtype], out.data_ptr(), q.K, s), "clq_mx4_dequantize")
    return out


def _product(q, qw, bias, experts):
    """Checks the operands of a product; the bias's type."""
    if not isinstance(q, MX4) or not isinstance(qw, MX4Weight):
        raise TypeError("the operands must be an MX4 and an MX4Weight")
    if q.K != qw.K:
        raise ValueError(f"inputs have {q.K} columns, weights {qw.K}")
    if q.block != qw.block:
        raise ValueError(f"inputs are rotated by blocks of {q.block}, weights by {qw.block}")
    if qw.experts != experts:
        raise ValueError(f"weights hold {qw.experts} experts, not {experts}")
    _same_device(q.codes.device, weights=qw.codes, bias=bias)
    if bias is None:
        return 0
    _dev(bias, "bias", _HALF)
    if bias.shape != ((qw.N,) if experts is None else (experts, qw.N)) or not bias.is_contiguous():
        raise ValueError("bias must be a contiguous [N] or [experts, N] tensor")
    return _TYPES[bias.dtype]


def _output(out, rows, N, dtype, device):
    if dtype not in _HALF:
        raise TypeError(f"dtype must be fp16 or bf16, got {dtype}")
    if out is None:   # rows on 16-byte boundaries
        ld = (N + 7) // 8 * 8
        out = torch.empty((rows, ld), dtype=dtype, device=device)
        return (out if ld == N else out[:, :N]), ld
    r, n, ld = _rows2d(out, "out", (dtype,))
    if r < rows or n != N:
        raise ValueError(f"out must be [{rows}, {N}]")
    _same_device(device, out=out)
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
    """Y = X . W^T + bias, fp16 or bf16 [M, N]."""
    bt = _product(q, qw, bias, None)
    if qw.gated:
        raise ValueError("gated weights go with clq_mx4_linear_mx4(act='swiglu')")
    with _On(q.codes.device, stream) as s:
        Y, ld = _output(out, q.rows, qw.N, dtype, q.codes.device)
        _check(_lib.clq_mx4_linear(q.codes.data_ptr(), q.scales.data_ptr(), qw.codes.data_ptr(), qw.scales.data_ptr(),
                                   _ptr(bias), bt, q.rows, qw.N, qw.K, _TYPES[dtype], Y.data_ptr(), ld, s),
               "clq_mx4_linear")
    return Y


def clq_mx4_linear_mx4(q, qw, bias=None, act=None, block=0, out=None, stream=None):
    """act(X . W^T + bias), rotated by blocks of `block` and quantized to MX4 without leaving
    fp32 in between: the input of the next product.  act: None, "gelu" (tanh form) or "swiglu"
    (gated weights, N / 2 columns)."""
    a = _act(act)
    bt = _product(q, qw, bias, None)
    with _On(q.codes.device, stream) as s:
        o = _buffers(out, q.rows, _columns(qw, a), q.codes.device, "clq_mx4_linear_mx4", block)
        _check(_lib.clq_mx4_linear_mx4(q.codes.data_ptr(), q.scales.data_ptr(), qw.codes.data_ptr(),
                                       qw.scales.data_ptr(), _ptr(bias), bt, q.rows, qw.N, qw.K, a, block,
                                       o.codes.data_ptr(), o.scales.data_ptr(), s), "clq_mx4_linear_mx4")
    return o


def clq_expert_route(logits, top_k, score="softmax", bias=None, groups=1, top_groups=1, renormalize=True, scale=1.0,
                     stream=None):
    """The top_k experts of each token and their weights: (ids int32 [T, top_k], weights fp32).
    logits: fp32, fp16 or bf16 [T, experts].  score: "softmax" or "sigmoid".  bias: fp32
    [experts], added for the ranking alone.  groups, top_groups: only the experts of the best
    top_groups of `groups` groups take part.  scale multiplies the weights."""
    _dev(logits, "logits", tuple(_TYPES))
    if logits.dim() != 2 or logits.stride(1) != 1 and logits.shape[1] != 1:
        raise ValueError("logits must be 2-D with unit column stride")
    if score not in _SCORES:
        raise ValueError(f"score must be 'softmax' or 'sigmoid', not {score!r}")
    T, E = logits.shape
    if bias is not None:
        _dev(bias, "bias", (torch.float32,))
        if bias.shape != (E,) or not bias.is_contiguous():
            raise ValueError(f"bias must be a contiguous fp32 [{E}] tensor")
        _same_device(logits.device, bias=bias)
    with _On(logits.device, stream) as s:
        ids = torch.empty((T, top_k), dtype=torch.int32, device=logits.device)
        weights = torch.empty((T, top_k), dtype=torch.float32, device=logits.device)
        _check(_lib.clq_expert_route(logits.data_ptr(), _TYPES[logits.dtype], max(logits.stride(0), E), T, E, top_k,
                                     _SCORES[score], _ptr(bias), groups, top_groups, int(renormalize), scale,
                                     ids.data_ptr(), weights.data_ptr(), s), "clq_expert_route")
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
    n = _lib.clq_expert_plan_rows(T, k, experts)
    if n == 0:
        raise ClqError(CLQ_ERR_SHAPE, "clq_expert_plan")
    nt, nw = _lib.clq_expert_plan_ints(experts), _lib.clq_expert_plan_workspace_bytes(T, k, experts)
    with _On(ids.device, stream) as s:
        # the tables, the rows and the sources in one buffer
        buf = torch.empty(nt + T * k + n, dtype=torch.int32, device=ids.device)
        tables, rows, source = buf.split_with_sizes((nt, T * k, n))
        ws = torch.empty(nw, dtype=torch.uint8, device=ids.device) if nw else None
        plan = ExpertPlan(T, k, experts, n, tables, rows.view(T, k), source)
        p = buf.data_ptr()
        _check(_lib.clq_expert_plan(ids.data_ptr(), T, k, experts, p, p + 4 * nt, p + 4 * (nt + T * k), _ptr(ws), nw,
                                    s), "clq_expert_plan")
    return plan


def clq_mx4_dispatch(X, plan, block=0, perm=None, out=None, stream=None):
    """clq_mx4_quantize of the tokens X [T, K] into the plan's rows, expert after expert."""
    T, K, ldx = _rows2d(X, "X")
    if T != plan.tokens:
        raise ValueError(f"X has {T} tokens, the plan {plan.tokens}")
    perm = _perm(perm, K)
    _same_device(X.device, perm=perm, plan=plan.tables)
    with _On(X.device, stream) as s:
        q = _buffers(out, plan.plan_rows, K, X.device, "clq_mx4_dispatch", block)
        _check(_lib.clq_mx4_dispatch(X.data_ptr(), _TYPES[X.dtype], ldx, _ptr(perm), T, plan.top_k, plan.experts, K,
                                     block, plan.tables.data_ptr(), plan.source.data_ptr(), q.codes.data_ptr(),
                                     q.scales.data_ptr(), s), "clq_mx4_dispatch")
    return q


def _plan_operands(q, plan):
    if q.rows != plan.plan_rows:
        raise ValueError(f"inputs have {q.rows} rows, the plan {plan.plan_rows}")
    _same_device(q.codes.device, plan=plan.tables)


def clq_mx4_experts(q, plan, qw, bias=None, dtype=None, out=None, stream=None):
    """Each row of the plan times its expert's weights: Y [plan.plan_rows, N], fp16 or bf16 (default:
    the bias's type, or fp16); rows past the last expert's are left as they were."""
    bt = _product(q, qw, bias, plan.experts)
    _plan_operands(q, plan)
    if qw.gated:
        raise ValueError("gated weights go with clq_mx4_experts_mx4(act='swiglu')")
    dtype = dtype or (torch.float16 if bias is None else bias.dtype)
    with _On(q.codes.device, stream) as s:
        Y, ld = _output(out, q.rows, qw.N, dtype, q.codes.device)
        _check(_lib.clq_mx4_experts(q.codes.data_ptr(), q.scales.data_ptr(), plan.tables.data_ptr(), plan.tokens,
                                    plan.top_k, plan.experts, qw.codes.data_ptr(), qw.scales.data_ptr(), _ptr(bias),
                                    bt, qw.N, qw.K, _TYPES[dtype], Y.data_ptr(), ld, s), "clq_mx4_experts")
    return Y


def clq_mx4_experts_mx4(q, plan, qw, bias=None, act=None, block=0, out=None, stream=None):
    """clq_mx4_linear_mx4 with each row times its expert's weights."""
    a = _act(act)
    bt = _product(q, qw, bias, plan.experts)
    _plan_operands(q, plan)
    with _On(q.codes.device, stream) as s:
        o = _buffers(out, q.rows, _columns(qw, a), q.codes.device, "clq_mx4_experts_mx4", block)
        _check(_lib.clq_mx4_experts_mx4(q.codes.data_ptr(), q.scales.data_ptr(), plan.tables.data_ptr(), plan.tokens,
                                        plan.top_k, plan.experts, qw.codes.data_ptr(), qw.scales.data_ptr(),
                                        _ptr(bias), bt, qw.N, qw.K, a, block, o.codes.data_ptr(),
                                        o.scales.data_ptr(), s), "clq_mx4_experts_mx4")
    return o


def clq_expert_combine(Y, plan, weights, out=None, stream=None):
    """out[t] = sum over the slots of weights[t, j] * Y[plan.rows[t, j]], in fp32, of Y's type."""
    r, N, ldy = _rows2d(Y, "Y")
    _dev(weights, "weights", (torch.float32,))
    if r < plan.plan_rows or weights.shape != plan.rows.shape or not weights.is_contiguous():
        raise ValueError("Y and weights must have the plan's rows and slots")
    _same_device(Y.device, weights=weights, plan=plan.tables)
    with _On(Y.device, stream) as s:
        o, ld = _output(out, plan.tokens, N, Y.dtype, Y.device)
        _check(_lib.clq_expert_combine(Y.data_ptr(), _TYPES[Y.dtype], ldy, plan.rows.data_ptr(), weights.data_ptr(),
                                       plan.tokens, plan.top_k, plan.experts, N, o.data_ptr(), ld, s),
               "clq_expert_combine")
    return o
