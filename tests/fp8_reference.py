"""Plain definitions, in 64 bits on the host, of the block-scaled 8-bit operators
(quantisation, products, the experts' products) and of the router with scores, with
bounds on what 32-bit sums and one fp16 rounding may add."""
import numpy as np

from mx4_reference import HALF, STEP32, expert_of_place, group, rounded  # noqa: F401

HALF32 = 2.0 ** -24
# the 127 magnitudes of e4m3
GRID = np.concatenate([np.arange(8) * 2.0 ** -9] + [np.arange(8, 16) * 2.0 ** (e - 10) for e in range(1, 16)])[:127]
MID = (GRID[1:] + GRID[:-1]) / 2


def quantize(x, rows=1):
    """fp16 [M][K] -> (codes [M][K] u8, scales [ceil(M/rows)][ceil(K/128)] float32)."""
    x = np.asarray(x, np.float16).astype(np.float64)
    M, K = x.shape
    R, G = -(-M // rows), -(-K // 128)
    b = np.zeros((R * rows, G * 128))
    b[:M, :K] = x
    b = b.reshape(R, rows, G, 128)
    finite = np.isfinite(b).all((1, 3))
    a = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0)).max((1, 3)), 0)
    f, e = np.frexp(np.where(a > 0, a, 448 / 512))  # a / 448 = f / 0.875 * 2^(e - 9)
    s = np.where(a > 0, np.exp2(e - 9.0 + (f > 0.875)), 1)
    assert (a <= 448 * s).all() and ((a > 224 * s) | (a == 0)).all()
    v = np.abs(np.where(finite[:, None, :, None], b, 0)) / s[:, None, :, None]
    low, high = np.searchsorted(MID, v, side="left"), np.searchsorted(MID, v, side="right")  # they differ at a tie
    codes = np.where(low % 2 == 0, low, high) + 128 * np.signbit(b)
    codes = np.where(finite[:, None, :, None], codes, 0).astype(np.uint8).reshape(R * rows, G * 128)[:M, :K]
    return codes, np.where(finite, s, np.nan).astype(np.float32)


def decoded(codes):
    c = np.asarray(codes)
    v = GRID[np.minimum(c & 127, 126)] * np.where(c & 128, -1.0, 1.0)
    return np.where((c & 127) == 127, np.nan, v)


def values(codes, scales, rows=128):
    """codes [..., N][K] with scales of blocks of `rows` rows and 128 columns."""
    s = np.repeat(np.repeat(np.asarray(scales, np.float64), rows, -2), 128, -1)
    return decoded(codes) * s[..., :codes.shape[-2], :codes.shape[-1]]


def quantized(x):
    return values(*quantize(x), rows=1)


def random_matrix(rng, *shape):
    """Codes of a normal distribution, scales near 2^-8 of any mantissa."""
    N, K = shape[-2:]
    flat = np.clip(rng.standard_normal(shape) * (448 / 4.2), -448, 448).astype(np.float16).reshape(-1, K)
    v = np.abs(flat.astype(np.float64))
    codes = (np.searchsorted(MID, v) + 128 * np.signbit(flat)).astype(np.uint8).reshape(shape)
    scales = np.exp2(rng.uniform(-9, -7, (*shape[:-2], -(-N // 128), -(-K // 128)))).astype(np.float32)
    return codes, scales


def additions(K, split=1):
    """Roundings of an addend on its way into an fp32 sum, each counted as a whole step
    (STEP32) of the sum of all magnitudes.  An instruction adds 128 products (7 levels;
    in two halves of 64, 6 and one more); its result is multiplied by the matrix's scale
    and added by one fused operation, at most once for each 128 columns; the sums of up
    to eight waves are added one by one, then those of `split` shares of K.  (A wave
    takes columns by 256, so that a lone one adds twice where K is short: one more.)"""
    return 7 + -(-K // 128) + 1 + 7 + split - 1


def largest8(v):
    """[rows][K] -> [rows][ceil(K/8)]: for each eight columns a bound on two to the
    exponent of the largest code, times its scale.  Codes below the normal ones count as
    2^-6, which is less than 2^-11 of the largest among the row's 128 wherever that one
    is 32 or more, as it is in these tests."""
    M, K = v.shape
    p = np.zeros((M, -(-K // 128) * 128))
    p[:, :K] = np.abs(np.where(np.isfinite(v), v, 0))
    group = p.reshape(M, -1, 128).max(-1)
    return np.maximum(p.reshape(M, -1, 8).max(-1), np.repeat(group, 16, 1) * 2.0 ** -11)


def product(a, w, n):
    """a [M][K] . w [N][K]^T and its bound: n additions, and what the matrix instruction
    drops.  It adds the products of eight neighbouring columns as whole numbers of
    2^(e - 13), e the largest sum of two exponents among them, each cut off towards
    zero: all but the largest lose less than 2^-13 of the largest's power of two."""
    return a @ w.T, n * STEP32 * (np.abs(a) @ np.abs(w).T) + 7 * 2.0 ** -13 * (largest8(a) @ largest8(w).T)


def gemm(x, w, residual=None, n=None):
    y, err = product(quantized(x), w, additions(w.shape[-1]) if n is None else n)
    if residual is not None:
        r = np.asarray(residual, np.float64)
        y, err = y + r, err + STEP32 * (np.abs(y) + np.abs(r))
    return y, rounded(y, err)


def gemm_mean_square(x, w, y):
    """The mean square that the errors of a product y have at most if they are
    independent: seven cut off products in eight, each of a third of the square of a
    whole cut (signs are random), one rounding to fp16, and a step of the 32-bit sums."""
    a = quantized(x)
    cut = 7 / 3 * 2.0 ** -26 * (largest8(a) ** 2 @ (largest8(w) ** 2).T)
    return np.mean(cut + (HALF * np.abs(y) + 2.0 ** -25) ** 2 + (STEP32 * (np.abs(a) @ np.abs(w).T)) ** 2)


def swiglu(x, wg, wu, offsets, rows, k, places=None, n=None):
    """h of some places (all that are there), and its bound.  silu has a slope of at
    most 1.1; its fast exponential rounds the product with log2 e and that constant
    (|g| steps together), its result, the sum with 1, the reciprocal and two products
    (one step each but the sum and the products, half: 4 steps at most)."""
    places = np.arange(offsets[-1]) if places is None else places
    n = additions(x.shape[1]) if n is None else n
    e_of = expert_of_place(offsets)[places]
    h, err = np.zeros((len(places), wg.shape[1])), np.zeros((len(places), wg.shape[1]))
    a = quantized(x[rows[places] // k]) if len(places) else np.zeros((0, x.shape[1]))
    for e in np.unique(e_of):
        at = e_of == e
        (g, eg), (u, eu) = product(a[at], wg[e], n), product(a[at], wu[e], n)
        with np.errstate(over="ignore"):
            s = g / (1 + np.exp(-g))
        h[at] = s * u
        err[at] = 1.1 * eg * (np.abs(u) + eu) + np.abs(s) * eu + (4 + np.abs(g)) * STEP32 * np.abs(h[at])
    return h, rounded(h, err)


def down(h, w, offsets, pos, weights, residual=None, tokens=None, n=None):
    """y of some tokens (all) and its bound: each slot is a fused product and sum, half
    a step of the magnitudes."""
    T, k = weights.shape
    tokens = np.arange(T) if tokens is None else tokens
    n = additions(h.shape[1]) if n is None else n
    e_of = expert_of_place(offsets)
    N = w.shape[1]
    y = np.zeros((len(tokens), N)) if residual is None else np.asarray(residual[tokens], np.float64)
    size, err = np.abs(y), np.zeros((len(tokens), N))
    place = pos.reshape(-1, k)[tokens]
    for j in range(k):
        for e in range(len(offsets) - 1):
            at = np.flatnonzero((place[:, j] >= 0) & (e_of[np.clip(place[:, j], 0, max(0, len(e_of) - 1))] == e)) if len(e_of) else np.zeros(0, int)
            if at.size:
                o, eo = product(quantized(h[place[at, j]]), w[e], n)
                p = weights[tokens[at], j].astype(np.float64)[:, None]
                y[at] += p * o
                err[at] += np.abs(p) * eo
                size[at] += np.abs(p) * np.abs(o)
    return y, rounded(y, err + k * HALF32 * size)


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0):
    """experts [T][k] and weights [T][k] of logits [T][E], fp16 or float32."""
    x = np.asarray(logits)
    most = float(np.finfo(x.dtype).max)
    x = x.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, most))
    T, E = x.shape
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if score == "sigmoid":
            s = 1 / (1 + np.exp(-x))
        else:
            top = x.max(-1, keepdims=True)
            p = np.exp(x - np.where(np.isfinite(top), top, 0))
            s = p / p.sum(-1, keepdims=True)
        s = s.astype(np.float32)
        c = s + np.asarray(0 if bias is None else bias, np.float32)
    assert c.dtype == np.float32
    c = np.where(np.isinf(x) | np.isnan(c), np.float32(-np.inf), c)
    size = E // groups
    experts, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        value = np.full(groups, -np.inf, np.float32)
        for g in range(groups):
            best = np.sort(c[t, g * size:(g + 1) * size])[::-1][:group_best]
            best = best[best > -np.inf]
            if best.size:
                value[g] = best.sum(dtype=np.float32)
        allowed = np.argsort(-value, kind="stable")[:top_groups]
        mine = np.where(np.isin(np.arange(E) // size, allowed), c[t], np.float32(-np.inf))
        order = np.argsort(-mine, kind="stable")[:k]
        order = order[mine[order] > -np.inf]
        experts[t, :order.size] = order
        w = s[t, order].astype(np.float64)
        total = w.sum() if renormalize else 1.0
        weights[t, :order.size] = w / total * np.float32(scale) if total > 0 else 0
    return experts, weights


def weight_bound(want):
    """The weights are made of the 32-bit scores in 64 bits and rounded once."""
    return 1.001 * HALF32 * np.abs(want) + 2.0 ** -149
