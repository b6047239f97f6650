"""Plain definitions, in 64 bits on the host, of the microscaled 4-bit (MXFP4)
operators: quantisation, products, routing and the experts' products, with
bounds on what 32-bit sums and one fp16 rounding may add."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
HALF = 2.0 ** -11   # half a step of fp16, relative
TINY = 2.0 ** -25   # half a step of the fp16 subnormals
STEP32 = 2.0 ** -23


def quantize(x):
    """fp16 [..., K] -> (codes [..., K/2] u8, scales [..., K/32] u8)."""
    x = np.asarray(x, np.float16).astype(np.float64)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    finite = np.isfinite(b).all(-1)
    a = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0)).max(-1), 0)
    e = np.frexp(np.where(a > 0, a, 1))[1] - 1 - 2
    scales = np.where(~finite, 255, np.where(a > 0, e + 127, 127)).astype(np.uint8)
    v = np.where(finite[..., None], b, 0) / np.exp2(np.where(a > 0, e, 0))[..., None]
    m = np.abs(v)[..., None]
    mid = (GRID[1:] + GRID[:-1]) / 2
    up = np.where(np.arange(7) % 2 == 1, m >= mid, m > mid)  # ties go to the even code
    codes = (up.sum(-1) + 8 * np.signbit(v)).astype(np.uint8)
    codes[~finite] = 0
    c = codes.reshape(x.shape)
    return c[..., 0::2] | c[..., 1::2] << 4, scales


def values(codes, scales):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def quantized(x):
    return values(*quantize(x))


def random_matrix(rng, *shape, spread=2):
    """Codes of a normal distribution, scales within 2^(-7 +- spread)."""
    K = shape[-1]
    codes, _ = quantize((rng.standard_normal(shape) * 2.2).astype(np.float16))
    return codes, rng.integers(120 - spread, 121 + spread, (*shape[:-1], K // 32)).astype(np.uint8)


def product(a, w):
    """a [M][K] . w [N][K]^T and the bound on an fp32 sum of the exact products:
    an instruction adds 128 products (a tree, 7 levels, and the alignment of its
    addends) and the accumulator, K / 128 of them follow one another, and up to
    16 partial sums are added: at most K / 128 + 32 roundings of each addend."""
    K = a.shape[-1]
    return a @ w.T, (K / 128 + 32) * STEP32 * (np.abs(a) @ np.abs(w).T)


def rounded(y, err):
    """The bound on fp16(y + err)."""
    return err + HALF * (np.abs(y) + err) + TINY


def gemm(x, w, residual=None):
    y, err = product(quantized(x), w)
    if residual is not None:
        r = np.asarray(residual, np.float64)
        y, err = y + r, err + STEP32 * (np.abs(y) + np.abs(r))
    return y, rounded(y, err)


def route(logits, k, renormalize=True):
    """experts [T][k], weights [T][k] of fp16 logits [T][E]."""
    x = np.asarray(logits, np.float16).astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, np.where(x == np.inf, 65504.0, x))
    T, E = x.shape
    order = np.argsort(-x, axis=-1, kind="stable")[:, :k]
    best = np.take_along_axis(x, order, -1)
    top = np.where(np.isfinite(best[:, :1]), best[:, :1], 0)
    p = np.exp(best - top)
    total = p.sum(-1, keepdims=True) if renormalize else np.exp(x - top).sum(-1, keepdims=True)
    weights = np.where(np.isfinite(best), p / np.where(total > 0, total, 1), 0)
    return np.where(np.isfinite(best), order, -1).astype(np.int32), weights


def group(experts, E):
    """offsets, rows, pos of experts [T][k]."""
    flat = np.asarray(experts).reshape(-1)
    key = np.where((flat < 0) | (flat >= E), E, flat)
    order = np.argsort(key, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])]).astype(np.int32)
    used = np.arange(flat.size) < offsets[-1]
    pos = np.empty(flat.size, np.int32)
    pos[order] = np.where(used, np.arange(flat.size), -1)
    return offsets, np.where(used, order, -1).astype(np.int32), pos


def expert_of_place(offsets):
    return np.repeat(np.arange(len(offsets) - 1), np.diff(offsets))


def swiglu(x, wg, wu, offsets, rows, k):
    """h of the places 0 .. offsets[-1], and its bound.  silu has a slope of at
    most 1.1; the fast exponential is off by a few steps and by the rounding of
    its argument, |g| steps."""
    a = quantized(x)
    n = offsets[-1]
    h, err = np.zeros((n, wg.shape[1])), np.zeros((n, wg.shape[1]))
    for e in range(len(offsets) - 1):
        at = slice(offsets[e], offsets[e + 1])
        mine = a[rows[at] // k]
        (g, eg), (u, eu) = product(mine, wg[e]), product(mine, wu[e])
        with np.errstate(over="ignore"):
            s = g / (1 + np.exp(-g))
        h[at] = s * u
        err[at] = 1.1 * eg * (np.abs(u) + eu) + np.abs(s) * eu + (8 + 2 * np.abs(g)) * STEP32 * np.abs(h[at])
    return h, rounded(h, err)


def down(h, w, offsets, pos, weights, residual=None):
    """y [T][N] and its bound."""
    T, k = weights.shape
    n = offsets[-1]
    o, eo = np.zeros((n, w.shape[1])), np.zeros((n, w.shape[1]))
    a = quantized(h[:n])
    for e in range(len(offsets) - 1):
        at = slice(offsets[e], offsets[e + 1])
        o[at], eo[at] = product(a[at], w[e])
    y = np.zeros((T, w.shape[1])) if residual is None else np.asarray(residual, np.float64).copy()
    err = np.zeros_like(y)
    size = np.abs(y)
    for t in range(T):
        for j in range(k):
            p = pos[t * k + j]
            if p >= 0:
                y[t] += float(weights[t, j]) * o[p]
                err[t] += abs(float(weights[t, j])) * eo[p]
                size[t] += abs(float(weights[t, j])) * np.abs(o[p])
    return y, rounded(y, err + (k + 1) * STEP32 * size)
