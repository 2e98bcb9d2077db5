"""Plain CPU oracle of the MX4 operators and of the expert layer (numpy, fp64).

Written from the definitions alone: MX4 codes are e2m1 values with one scale
2^e for 32 values, e = max(floor(log2(max|x|)) - 2, -126), rounded to nearest with
ties to the even code and saturated at 6.  The rotation runs in fp32 in the library's
documented stage order (h = 1, 2, ...), where a rounding can decide a code.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotate(x, block, perm=None):
    """FWHT_block(gather(x, perm)) in fp32; x: [..., K] of any float type."""
    v = np.asarray(x, dtype=np.float32)
    if perm is not None:
        v = v[..., np.asarray(perm)]
    h = 1
    with np.errstate(over="ignore", invalid="ignore"):
        while h < block:
            p = v.reshape(*v.shape[:-1], -1, 2, h)
            v = np.stack((p[..., 0, :] + p[..., 1, :], p[..., 0, :] - p[..., 1, :]), axis=-2).reshape(v.shape)
            h *= 2
    return v


def exponents(v):
    """The scale exponent of each 32 values (last axis); 128 where a group is not finite."""
    g = np.abs(np.asarray(v, dtype=np.float64)).reshape(*v.shape[:-1], -1, 32).max(-1)
    bad = ~np.isfinite(g)
    e = np.frexp(np.where(bad, 1.0, g))[1] - 3
    e = np.where(g == 0, -126, np.maximum(e, -126))
    return np.where(bad, 128, e)


def on_grid(v, e):
    """v / 2^e rounded to the grid, times 2^e (e: one for 32 values)."""
    s = np.ldexp(1.0, np.repeat(np.where(e == 128, 0, e), 32, axis=-1))
    a = np.abs(np.asarray(v, dtype=np.float64)) / s
    lo = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 7)
    hi = np.minimum(lo + 1, 7)
    with np.errstate(invalid="ignore"):
        up, down = GRID[hi] - a, a - GRID[lo]
        pick = np.where(up < down, hi, np.where(up > down, lo, np.where(lo % 2 == 0, lo, hi)))
    out = np.copysign(GRID[pick], v) * s
    return np.where(np.repeat(e == 128, 32, axis=-1), np.nan, out)


def quantize(x, block=0, perm=None, divide=1.0):
    """The values that the quantizer's codes and scales stand for."""
    v = rotate(x, block, perm).astype(np.float64) / divide
    return on_grid(v, exponents(v))


def gelu(h):
    return 0.5 * h * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (h + 0.044715 * h ** 3)))


def activate(h, act):
    if act == "gelu":
        return gelu(h)
    if act == "swiglu":
        f = h.shape[-1] // 2
        return h[..., :f] / (1.0 + np.exp(-h[..., :f])) * h[..., f:]
    return h


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, renormalize=True, scale=1.0):
    """(ids, weights, ranks) in fp64; ties to the lower index."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "softmax":
            m = x.max(-1, keepdims=True)
            p = np.where(np.isneginf(m), 0.0, np.exp(x - np.where(np.isneginf(m), 0.0, m)))
            s = p / np.where(np.isneginf(m), 1.0, p.sum(-1, keepdims=True))
        else:
            s = 1.0 / (1.0 + np.exp(-x))
    rank = x.copy() if bias is None and groups == 1 else s + (0.0 if bias is None else np.asarray(bias, np.float64))
    if groups > 1:
        g = rank.reshape(T, groups, -1)
        best = np.sort(g, -1)[..., ::-1][..., :2].sum(-1)
        order = np.argsort(-best, -1, kind="stable")[:, :top_groups]
        keep = np.zeros((T, groups), bool)
        np.put_along_axis(keep, order, True, -1)
        open_ = np.repeat(keep, E // groups, -1)
    else:
        open_ = np.ones((T, E), bool)
    # (an open expert goes before a closed one, whatever its rank)
    key = np.lexsort((np.broadcast_to(np.arange(E), (T, E)), -rank, ~open_), axis=-1)
    ids = key[:, :k]
    w = np.take_along_axis(s, ids, -1)
    if renormalize:
        total = w.sum(-1, keepdims=True)
        w = np.where(total > 0, w / np.where(total > 0, total, 1.0), 0.0)
    return ids.astype(np.int32), w * scale, np.where(open_, rank, -np.inf)


def plan(ids, E):
    """(counts, rows, source of the rows in use)."""
    T, k = ids.shape
    flat = ids.reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(E)], np.int64)
    units = (counts + 31) // 32
    first = 32 * (np.cumsum(units) - units)
    rows = np.full(flat.shape, -1, np.int64)
    source = np.full(32 * units.sum(), -1, np.int64)
    for e in range(E):
        at = np.nonzero(flat == e)[0]
        rows[at] = first[e] + np.arange(len(at))
        source[rows[at]] = at // k
    return counts, rows.reshape(T, k), source
