"""Python binding of the operators around the 8-bit linears of a transformer block
(``include/clq_block.h``).

Argument marshalling only, in the manner of the package's other entry points:

    clq_rms_norm(X, weight=None, residual=None, eps=1e-6)            -> Y, or (Y, sum)
    clq_rms_norm_act8(X, block, weight=None, residual=None, eps=1e-6, perm=None)
                                                                     -> (Xq8, x_scale), or (Xq8, x_scale, sum)
    clq_quantize_act8(X, block, perm=None)                           -> (Xq8, x_scale)
    clq_dequantize_act8(Xq8, x_scale, K, dtype=torch.float16)        -> values
    clq_rope_freqs(axes, theta=10000.0, device="cuda")               -> freqs
    clq_rope_axes(X, positions, freqs, axes, interleaved=True, inverse=False, weight=None) -> Y
    clq_a8_linear_act(Xq8, x_scale, qw, bias=None, act=None, gate=None, residual=None) -> Y

Every call enqueues on the current stream, or on `stream`; what it allocates belongs
to that stream.  Nothing here has a gradient of its own: the package is post-training quantization.
"""
import ctypes
import functools

import torch

from . import CLQ_ERR_ARG, CLQ_ERR_SHAPE, ClqError, _check, _lib, _raw_stream
from .mx4 import _HALF, _TYPES, _current_device, _dev, _elsewhere, _gather, _meet, _output, _row_bytes, _rows2d, _together

_i64, _i32, _f32, _p = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p
_SIGNATURES = {
    "clq_rms_norm": (_i32, [_p, _i32, _i64, _p, _i32, _i64, _p, _i32, _i64, _f32, _i64, _i64, _p, _i32, _i64, _p, _i64,
                            _p]),
    "clq_rms_norm_act8": (_i32, [_p, _i32, _i64, _p, _i32, _i64, _p, _i32, _i64, _f32, _p, _i64, _i64, _i32, _p, _p, _p,
                                 _i64, _p]),
    "clq_quantize_act8": (_i32, [_p, _i32, _i64, _p, _i64, _i64, _i32, _p, _p, _p]),
    "clq_dequantize_act8": (_i32, [_p, _p, _i64, _i64, _i32, _p, _i64, _p]),
    "clq_rope_axes": (_i32, [_p, _i32, _i64, _i64, _p, _i32, _i64, _p, _p, _i32, _i32, _i32, _p, _i32, _i64, _f32, _i64,
                             _i64, _i64, _p, _i64, _i64, _p]),
    "clq_a8_linear_act": (_i32, [_p, _p, _p, _p, _i32, _p, _i32, _i32, _p, _i32, _i64, _p, _i64, _i64, _i64, _i64, _i32, _p,
                                 _i64, _p]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    getattr(_lib, _name).restype = _res
    getattr(_lib, _name).argtypes = _args

BLOCK_EXPORTS = tuple(_SIGNATURES)
__all__ = ["BLOCK_EXPORTS", "clq_rope_freqs", *BLOCK_EXPORTS]

_POSITIONS = {torch.int32: 0, torch.float32: 1}
_F64, _F32, _U8 = (torch.float64,), (torch.float32,), (torch.uint8,)
_NONE, _NO_RESIDUAL = (None, 0, 1), (None, 0, 0)
_ACTS = {None: 0, "none": 0, "gelu": 1, "silu": 3}
_WIDEST = 16384   # columns of the norm's rows and of those that are quantized from 32 bits


def _flat_bytes(t):
    n = t.numel() * t.element_size()
    return t.data_ptr(), 1, n, n


def _apart(out, *inputs):
    """An output of the caller's must not lie in what the launch reads: where the spans they lie in meet, pieces
    at one distance are compared piece by piece."""
    at, n, pitch, width = out
    end = at + (n - 1) * pitch + width
    for x in inputs:
        if x[0] >= end or x[0] + (x[1] - 1) * x[2] + x[3] <= at:
            continue
        a, b = ((p[0], 1, 1, p[1] * p[3]) if p[1] == 1 or p[2] == p[3] else p for p in (out, x))
        if a[1] != 1 and b[1] != 1 and a[2] != b[2] or _meet(a, b):
            raise ValueError("the output overlaps an input")


def _matrix(X, name):
    """_rows2d of any of the three types, and the type as the C calls take it."""
    if not isinstance(X, torch.Tensor) or not X.is_cuda or X.dtype not in _TYPES or X.dim() != 2:
        return *_rows2d(X, name, _TYPES), None   # (which says what is wrong)
    (M, K), (ld, step) = X.shape, X.stride()
    if step != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    return M, K, ld if M > 1 else (K + 7) & ~7, _TYPES[X.dtype]   # (a single row has no stride of its own)


def _modulation(w, name, K, M, device):
    """Pointer, type and samples of a [K] or [samples, K] matrix (None: none)."""
    if w is None:
        return _NONE
    t = _dev(w, name, _TYPES).dtype
    shape = w.shape
    if len(shape) not in (1, 2) or shape[-1] != K or not w.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{K}] or [samples, {K}] tensor")
    samples = 1 if len(shape) == 1 else shape[0]
    if samples < 1 or M % samples:
        raise ValueError(f"{name} has {samples} samples, which do not divide {M} rows")
    if w.device != device:
        _together(device, name, w)
    return w.data_ptr(), _TYPES[t], samples


def _in_place(out, t, ld_out, ld):
    """Whether an output is that very matrix."""
    return out.data_ptr() == t.data_ptr() and ld_out == ld and out.dtype == t.dtype


def _norm_operands(X, weight, residual, sum_out):
    """Checks what both forms of the norm share; (rows, columns, stride, type, device, weight, residual), the
    last two as the C call takes them."""
    M, K, ldx, xt = _matrix(X, "X")
    device = X.device
    w = _NONE if weight is None else _modulation(weight, "weight", K, M, device)
    if residual is None:
        if sum_out is not None:
            raise ValueError("there is no sum without a residual")
        return M, K, ldx, xt, device, w, _NO_RESIDUAL
    r, k, ldr, rt = _matrix(residual, "residual")
    if r != M or k != K:
        raise ValueError(f"residual must be [{M}, {K}]")
    if residual.device != device:
        _together(device, "residual", residual)
    if sum_out is not None:
        _check_sum(X, residual, sum_out, M, K, ldx, ldr, weight)
    return M, K, ldx, xt, device, w, (residual.data_ptr(), rt, ldr)


def _check_sum(X, residual, sum_out, M, K, ldx, ldr, weight):
    s, n, lds = _rows2d(sum_out, "sum_out", (residual.dtype,))
    if s != M or n != K:
        raise ValueError(f"sum_out must be [{M}, {K}]")
    if sum_out.device != X.device:
        _together(X.device, "sum_out", sum_out)
    at, reads = _row_bytes(sum_out, M, K, lds), [_row_bytes(X, M, K, ldx)]
    if not _in_place(sum_out, residual, lds, ldr):
        reads.append(_row_bytes(residual, M, K, ldr))
    if weight is not None:
        reads.append(_flat_bytes(weight))
    _apart(at, *reads)


def _norm_inputs(weight, residual, M, K, ldr):
    """What a norm's output must not lie in, X apart."""
    reads = []
    if weight is not None:
        reads.append(_flat_bytes(weight))
    if residual is not None:
        reads.append(_row_bytes(residual, M, K, ldr))
    return reads


def clq_rms_norm(X, weight=None, residual=None, eps=1e-6, dtype=None, out=None, sum_out=None, stream=None):
    """Y = s / sqrt(mean(s^2) + eps) * weight with s = X + residual, per row.  X: fp16, bf16 or fp32 [M, K], any
    row stride that is a multiple of 8.  weight: [K], or [samples, K] for rows of that many equal samples.
    residual: fp16, bf16 or fp32 [M, K]; the sum comes back too, in its type (sum_out: where, the residual
    itself included).  dtype: of Y (X's by default).  out: where, X itself included.  Squares are summed in
    fp32: rows whose sum of them reaches 2^128 come out as zeros."""
    M, K, ldx, xt, device, w, r = _norm_operands(X, weight, residual, sum_out)
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_rms_norm(X, weight, residual, eps, dtype, out, sum_out)
    if dtype is None:
        dtype = X.dtype if out is None else out.dtype
    if out is None and dtype in _TYPES:
        Y, ldy = torch.empty(M, K, dtype=dtype, device=device), K
    else:
        Y, ldy = _output(out, M, K, dtype, device)
        reads = _norm_inputs(weight, residual, M, K, r[2])
        if not _in_place(Y, X, ldy, ldx):
            reads.append(_row_bytes(X, M, K, ldx))
        if sum_out is not None:
            reads.append(_row_bytes(sum_out, M, K, sum_out.stride(0) if M > 1 else K))
        _apart(_row_bytes(Y, M, K, ldy), *reads)
    S, s, lds = _sum(residual, sum_out, M, K, device)
    status = _lib.clq_rms_norm(X.data_ptr(), xt, ldx, r[0], r[1], r[2], w[0], w[1], w[2], eps, M, K, Y.data_ptr(),
                               _TYPES[dtype], ldy, s, lds, _raw_stream(i))
    if status:
        _check(status, "clq_rms_norm")
    return Y if S is None else (Y, S)


def _sum(residual, sum_out, M, K, device):
    """Where the sum goes: a tensor, its address and row stride."""
    if residual is None:
        return None, None, 0
    if sum_out is None:
        S = torch.empty(M, K, dtype=residual.dtype, device=device)
        return S, S.data_ptr(), K
    return sum_out, sum_out.data_ptr(), sum_out.stride(0) if M > 1 else K


def _codes(M, K, device, out, scale_out, reads, where):
    """Buffers of 8-bit codes and their scales: the caller's, checked against what the call reads, or new ones."""
    if not 0 < M < 2147483648 or not 64 <= K <= _WIDEST or K & 63:
        raise ClqError(CLQ_ERR_SHAPE, where)
    n = (M + 31) // 32 * 32 * K
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, device=device)
    else:
        if _dev(out, "out", (torch.uint8,)).numel() < n or not out.is_contiguous():
            raise ValueError("the output's buffer is too small")
        _together(device, "out", out)
        _apart((out.data_ptr(), 1, n, n), *reads)
    if scale_out is None:
        scale_out = torch.empty(M, dtype=torch.float32, device=device)
    else:
        if _dev(scale_out, "scale_out", _F32).dim() != 1 or scale_out.numel() < M or not scale_out.is_contiguous():
            raise ValueError(f"scale_out must be a contiguous tensor of at least {M} scales")
        _together(device, "scale_out", scale_out)
        scale_out = scale_out if scale_out.numel() == M else scale_out[:M]
        _apart((scale_out.data_ptr(), 1, 4 * M, 4 * M), (out.data_ptr(), 1, n, n), *reads)
    return out, scale_out


def clq_rms_norm_act8(X, block, weight=None, residual=None, eps=1e-6, perm=None, out=None, scale_out=None,
                      sum_out=None, stream=None):
    """The norm of clq_rms_norm rotated by blocks of `block` (after gathering its columns by `perm`) and
    quantized to 8 bits a value with one scale a row, without a rounding in between: what
    clq_rotate_quant_act8 returns, (Xq8 uint8 [clq_act8_bytes(M, K)], x_scale fp32 [M]), and with a
    residual the sum."""
    M, K, ldx, xt, device, w, r = _norm_operands(X, weight, residual, sum_out)
    g = None if perm is None else _gather(perm, K, device)
    if perm is not None and sum_out is not None:
        _apart(_row_bytes(sum_out, M, K, sum_out.stride(0) if M > 1 else K), _flat_bytes(perm))
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_rms_norm_act8(X, block, weight, residual, eps, perm, out, scale_out, sum_out)
    if out is None and scale_out is None:
        q, xs = _codes(M, K, device, None, None, (), "clq_rms_norm_act8")
    else:
        reads = _norm_inputs(weight, residual, M, K, r[2])
        reads.append(_row_bytes(X, M, K, ldx))
        if perm is not None:
            reads.append(_flat_bytes(perm))
        if sum_out is not None:
            reads.append(_row_bytes(sum_out, M, K, sum_out.stride(0) if M > 1 else K))
        q, xs = _codes(M, K, device, out, scale_out, reads, "clq_rms_norm_act8")
    S, s, lds = _sum(residual, sum_out, M, K, device)
    status = _lib.clq_rms_norm_act8(X.data_ptr(), xt, ldx, r[0], r[1], r[2], w[0], w[1], w[2], eps, g, M, K, block,
                                    q.data_ptr(), xs.data_ptr(), s, lds, _raw_stream(i))
    if status:
        _check(status, "clq_rms_norm_act8")
    return (q, xs) if S is None else (q, xs, S)


def clq_quantize_act8(X, block, perm=None, out=None, scale_out=None, stream=None):
    """clq_rotate_quant_act8 of fp16, bf16 or fp32 activations [M, K] (any row stride that is a multiple of 8):
    the same codes and scales for finite fp16 values."""
    M, K, ldx, xt = _matrix(X, "X")
    device = X.device
    g = None if perm is None else _gather(perm, K, device)
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_quantize_act8(X, block, perm, out, scale_out)
    q, xs = _codes(M, K, device, out, scale_out,
                   () if out is None and scale_out is None else (_row_bytes(X, M, K, ldx), *(() if perm is None else (_flat_bytes(perm),))),
                   "clq_quantize_act8")
    status = _lib.clq_quantize_act8(X.data_ptr(), xt, ldx, g, M, K, block, q.data_ptr(), xs.data_ptr(), _raw_stream(i))
    if status:
        _check(status, "clq_quantize_act8")
    return q, xs


def _rows8(Xq8, x_scale, K):
    """Rows of 8-bit activations, checked."""
    _dev(Xq8, "Xq8", _U8)
    _dev(x_scale, "x_scale", _F32)
    M = x_scale.shape[0] if x_scale.dim() == 1 else 0
    if M < 1 or not x_scale.is_contiguous():
        raise ValueError("x_scale must be a contiguous [M] tensor")
    if Xq8.numel() < (M + 31) // 32 * 32 * K or not Xq8.is_contiguous():
        raise ValueError("Xq8 must be the contiguous buffer of 8-bit codes of these rows and K")
    if x_scale.device != Xq8.device:
        _together(Xq8.device, "x_scale", x_scale)
    return M


def clq_dequantize_act8(Xq8, x_scale, K, dtype=torch.float16, out=None, stream=None):
    """The values that 8-bit activations stand for (still rotated): fp16, bf16 or fp32 [M, K], M =
    len(x_scale)."""
    M = _rows8(Xq8, x_scale, K)
    device = Xq8.device
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_dequantize_act8(Xq8, x_scale, K, dtype, out)
    if out is None and dtype in _TYPES and not K & 7:
        o, ld = torch.empty(M, K, dtype=dtype, device=device), K
    else:
        o, ld = _output(out, M, K, dtype, device)
        _apart(_row_bytes(o, M, K, ld), _flat_bytes(Xq8), _flat_bytes(x_scale))
    status = _lib.clq_dequantize_act8(Xq8.data_ptr(), x_scale.data_ptr(), M, K, _TYPES[dtype], o.data_ptr(), ld, _raw_stream(i))
    if status:
        _check(status, "clq_dequantize_act8")
    return o


@functools.lru_cache(maxsize=64)
def _pair_ends(axes):
    """Pairs of the axes so far, from the columns each axis turns (a tuple)."""
    if not 1 <= len(axes) <= 4 or any(int(d) != d or d < 2 or d % 2 for d in axes):
        raise ValueError("axes must be one to four positive even numbers of columns")
    ends, n = (_i32 * len(axes))(), 0
    for j, d in enumerate(axes):
        n += int(d) // 2
        ends[j] = n
    return ends, n, ctypes.addressof(ends), len(axes)


def clq_rope_freqs(axes, theta=10000.0, device="cuda"):
    """Radians a position for each pair: an axis of d columns has theta^(-2 j / d), j = 0 .. d / 2 - 1
    (fp64 [sum(axes) / 2])."""
    _pair_ends(tuple(axes))
    if not 0 < theta < float("inf"):
        raise ValueError(f"theta must be positive and finite, not {theta}")
    return torch.cat([float(theta) ** (-torch.arange(0, d, 2, dtype=torch.float64, device=device) / d) for d in axes])


def _head_strides(X, name, types):
    """Rows, heads, head width, row and head strides of [M, heads, D]."""
    _dev(X, name, types)
    if X.dim() != 3 or (X.stride(2) != 1 and X.shape[2] != 1):
        raise ValueError(f"{name} must be [rows, heads, D] with unit column stride")
    M, H, D = X.shape
    ld, lh = X.stride(0), X.stride(1)
    # (a single row or head has no stride of its own; torch gives such a view any)
    lh = D if H == 1 else lh
    return M, H, D, (max(H * lh, D) + 7) & ~7 if M == 1 else ld, lh


def _head_bytes(X, M, H, D, ld, lh):
    size = X.element_size()
    if ld >= lh or H == 1:
        return X.data_ptr(), M, ld * size, ((H - 1) * lh + D) * size
    return X.data_ptr(), H, lh * size, ((M - 1) * ld + D) * size


def _heads_meet(at, M, ld, H, lh, D):
    """Whether two sets of M rows of H heads of one spacing meet, the second `at` behind the first."""
    (n, outer), (m, inner) = ((M, ld), (H, lh)) if ld >= lh else ((H, lh), (M, ld))
    span = (m - 1) * inner + D
    for i in range(max(1 - n, (-at - span) // outer + 1), min(n - 1, (span - 1 - at) // outer) + 1):
        j = max(1 - m, -((at + i * outer + D - 1) // inner))   # the first whose end lies behind the other's start
        if j < m and at + i * outer + j * inner < D:
            return True
    return False


def clq_rope_axes(X, positions, freqs, axes, interleaved=True, inverse=False, weight=None, eps=1e-6, out=None,
                  stream=None):
    """Turns the first sum(axes) columns of each head by its row's position on each axis.  X: fp16 or bf16
    [rows, heads, D], strides multiples of 8 (columns of a wider projection, queries and keys together).
    positions: int32 or fp32 [tokens, len(axes)], for rows that repeat those tokens (a batch).  freqs: fp64
    [sum(axes) / 2] radians a position (clq_rope_freqs).  interleaved: pairs are neighbours; otherwise a column
    pairs with the one half of the turned columns on.  inverse: by the opposite angles.  weight: [D] or
    [heads, D] of an RMS norm of each head ahead of the turn.  out: where, X itself included."""
    M, H, D, ldx, lhx = _head_strides(X, "X", _HALF)
    device = X.device
    _, n, ends, na = _pair_ends(tuple(axes))
    pt = _dev(positions, "positions", _POSITIONS).dtype
    shape = positions.shape
    if len(shape) != 2 or shape[1] != na or not positions.is_contiguous():
        raise ValueError(f"positions must be a contiguous [tokens, {na}] tensor")
    tokens = shape[0]
    if tokens < 1 or M % tokens:
        raise ValueError(f"positions of {tokens} tokens do not repeat over {M} rows")
    if _dev(freqs, "freqs", _F64).shape != (n,) or not freqs.is_contiguous():
        raise ValueError(f"freqs must be a contiguous fp64 [{n}] tensor")
    if 2 * n > D:
        raise ValueError(f"the axes turn {2 * n} columns, a head has {D}")
    if positions.device != device or freqs.device != device:
        raise ValueError(f"positions and freqs are on {positions.device} and {freqs.device}, not on {device}")
    w, wt, wh = None, 0, 1
    if weight is not None:
        _dev(weight, "weight", _TYPES)
        if weight.shape not in ((D,), (H, D)) or not weight.is_contiguous():
            raise ValueError(f"weight must be a contiguous [{D}] or [{H}, {D}] tensor")
        _together(device, "weight", weight)
        w, wt, wh = weight.data_ptr(), _TYPES[weight.dtype], 1 if weight.dim() == 1 else H
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_rope_axes(X, positions, freqs, axes, interleaved, inverse, weight, eps, out)
    if out is None:
        Y, ldy, lhy = torch.empty(M, H, D, dtype=X.dtype, device=device), H * D, D
    else:
        m, h, d, ldy, lhy = _head_strides(out, "out", (X.dtype,))
        if (m, h, d) != (M, H, D):
            raise ValueError(f"out must be [{M}, {H}, {D}]")
        _together(device, "out", out)
        Y, at = out, _head_bytes(out, M, H, D, ldy, lhy)
        if ldy == ldx >= D and lhy == lhx >= D:   # (others are refused by the call)
            if not _in_place(Y, X, ldy, ldx) and _heads_meet((Y.data_ptr() - X.data_ptr()) // 2, M, ldx, H, lhx, D):
                raise ValueError("the output overlaps an input")
        else:
            _apart(at, _head_bytes(X, M, H, D, ldx, lhx))
        _apart(at, _flat_bytes(positions), _flat_bytes(freqs), *(() if weight is None else (_flat_bytes(weight),)))
    status = _lib.clq_rope_axes(X.data_ptr(), _TYPES[X.dtype], ldx, lhx, positions.data_ptr(), _POSITIONS[pt], tokens,
                                freqs.data_ptr(), ends, na, 1 if interleaved else 0, 1 if inverse else 0, w, wt, wh, eps, M,
                                H, D, Y.data_ptr(), ldy, lhy, _raw_stream(i))
    if status:
        _check(status, "clq_rope_axes")
    return Y


def _result_type(act, N):
    """Of a result whose caller names none.  Activated values go to the next linear's quantizer: rounded to 16 bits
    ahead of it their codes part from the formula's next to a border (an MLP of 8192 x 1152 -> 4608 -> 1152 is
    then 4.3 to 4.8e-4 off its definition instead of 3.0e-4).  Rows that the quantizer takes in 16 bits only stay
    16 bits."""
    return torch.float32 if act not in (None, "none") and N <= _WIDEST else torch.float16


def clq_a8_linear_act(Xq8, x_scale, qw, bias=None, act=None, gate=None, residual=None, dtype=None, out=None, stream=None):
    """clq_a8_linear with an epilogue: Y = residual + gate * act(X . W^T + bias), fp32 throughout and rounded
    once.  act: None, "gelu" (tanh form) or "silu".  gate: [N], or [samples, N] for rows of that many equal
    samples.  residual: of Y's type [M, N].  dtype: of Y; by default that of `out` or of the residual, else fp32
    behind an activation (what clq_rotate_quant_act8 takes unrounded: N <= 16384) and fp16 otherwise.  out: where,
    the residual itself included."""
    N, K, bits, wq, ws, device = qw.N, qw.K, qw.bits, qw.wq, qw.w_scale, Xq8.device
    M = _rows8(Xq8, x_scale, K)
    if bits not in (4, 8):
        raise ClqError(CLQ_ERR_ARG, "clq_a8_linear_act")
    if wq.dtype != torch.uint8 or ws.dtype != torch.float32 or not wq.is_contiguous() or not ws.is_contiguous() or \
            wq.numel() < (N + 63) // 64 * 64 * K * bits // 8 or ws.numel() < N:   # (rows are padded to 64)
        raise ValueError("the weights' buffers are not those of their N and K")
    if act not in _ACTS:
        raise ValueError(f"act must be None, 'gelu' or 'silu', not {act!r}")
    if wq.device != device or ws.device != device:
        raise ValueError(f"weights are on {wq.device}, not on {device}")
    b, bt = None, 0
    if bias is not None:
        bt = _TYPES[_dev(bias, "bias", _HALF).dtype]
        if bias.shape != (N,) or not bias.is_contiguous():
            raise ValueError(f"bias must be a contiguous [{N}] tensor")
        if bias.device != device:
            _together(device, "bias", bias)
        b = bias.data_ptr()
    g, gt, samples = _modulation(gate, "gate", N, M, device)
    if dtype is None:
        given = out if out is not None else residual
        dtype = given.dtype if given is not None else _result_type(act, N)
    r, ldr = None, 0
    if residual is not None:
        rows, columns, ldr = _rows2d(residual, "residual", (dtype,))
        if (rows, columns) != (M, N):
            raise ValueError(f"residual must be [{M}, {N}]")
        _together(device, "residual", residual)
        r = residual.data_ptr()
    i = device.index
    if stream is not None or _current_device() != i:
        with _elsewhere(device, stream):
            return clq_a8_linear_act(Xq8, x_scale, qw, bias, act, gate, residual, dtype, out)
    Y, ld = _output(out, M, N, dtype, device)
    if out is not None:
        at = _row_bytes(Y, M, N, ld)
        if residual is not None and not _in_place(Y, residual, ld, ldr):
            _apart(at, _row_bytes(residual, M, N, ldr))
        _apart(at, *(_flat_bytes(t) for t in (Xq8, x_scale, wq, ws, bias, gate) if t is not None))
    status = _lib.clq_a8_linear_act(Xq8.data_ptr(), x_scale.data_ptr(), wq.data_ptr(), ws.data_ptr(), bits, b, bt, _ACTS[act],
                                    g, gt, samples, r, ldr, M, N, K, _TYPES[dtype], Y.data_ptr(), ld, _raw_stream(i))
    if status:
        _check(status, "clq_a8_linear_act")
    return Y
