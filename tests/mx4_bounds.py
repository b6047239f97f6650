"""Bounds on the 4-bit products by the form that runs them, for a sample of rows,
beside their 64-bit values (mx4_reference.py has the operators themselves)."""
import numpy as np

import mx4_reference as ref
from mx4_reference import HALF, STEP32, TINY

HALF32 = 2.0 ** -24


def additions(K, form, split=1):
    """Roundings of an addend on its way into an fp32 sum, each counted as a whole
    step (STEP32) of the sum of all magnitudes.  "tile": an instruction adds 64
    products (a tree of 6 levels) to the accumulator, ceil(K / 64) of them in whole
    words of 512 columns a share follow one another, then `split` parts are added.
    "stream": 128 products (7 levels), eight waves share the chunks of 256 columns,
    and their sums are added."""
    if form.startswith("tile"):
        return 6 + 8 * -(-(-(-K // 512)) // split) + split - 1
    return 7 + 2 * -(-(-(-K // 256)) // 8) + 7


def product(a, w, n):
    """a [M][K] . w [N][K]^T and the bound of n additions."""
    return a @ w.T, n * STEP32 * (np.abs(a) @ np.abs(w).T)


def rounded(y, err):
    """The bound on fp16(y + err): half a step."""
    return err + HALF * (np.abs(y) + err) + TINY


def swiglu(x, wg, wu, offsets, rows, k, places, n):
    """h of some places and its bound.  silu has a slope of at most 1.1; its fast
    exponential rounds the product with log2 e and that constant (|g| steps
    together), its result, the sum with 1, the reciprocal and two products (one
    step each but the sum and the products, half: 4 steps at most)."""
    e_of = ref.expert_of_place(offsets)[places]
    h, err = np.zeros((len(places), wg.shape[1])), np.zeros((len(places), wg.shape[1]))
    a = ref.quantized(x[rows[places] // k])
    for e in np.unique(e_of):
        at = e_of == e
        (g, eg), (u, eu) = product(a[at], wg[e], n), product(a[at], wu[e], n)
        with np.errstate(over="ignore"):
            s = g / (1 + np.exp(-g))
        h[at] = s * u
        err[at] = 1.1 * eg * (np.abs(u) + eu) + np.abs(s) * eu + (4 + np.abs(g)) * STEP32 * np.abs(h[at])
    return h, rounded(h, err)


def down(h, w, offsets, pos, weights, residual, tokens, n):
    """y of some tokens and its bound: each slot is a fused product and sum, half a
    step of the magnitudes."""
    k = weights.shape[1]
    e_of = ref.expert_of_place(offsets)
    N = w.shape[1]
    y = np.zeros((len(tokens), N)) if residual is None else np.asarray(residual[tokens], np.float64)
    size, err = np.abs(y), np.zeros((len(tokens), N))
    place = pos.reshape(-1, k)[tokens]
    for j in range(k):
        for e in range(len(offsets) - 1):
            at = np.flatnonzero((place[:, j] >= 0) & (e_of[np.clip(place[:, j], 0, max(0, len(e_of) - 1))] == e)) if len(e_of) else np.zeros(0, int)
            if at.size:
                o, eo = product(ref.quantized(h[place[at, j]]), w[e], n)
                p = weights[tokens[at], j].astype(np.float64)[:, None]
                y[at] += p * o
                err[at] += np.abs(p) * eo
                size[at] += np.abs(p) * np.abs(o)
    return y, rounded(y, err + k * HALF32 * size)


def route_weights(want, E, renormalize):
    """The bound on the router's weights where the differences of the scores are
    exact: exp is off by one step above and below the line; a lane adds up to E / 16
    scores (a power of two), 16 lanes in four levels (with renormalisation only
    these), half a step each, as is the division."""
    lane = 1
    while 16 * lane < E:
        lane *= 2
    adds = 4 if renormalize else lane + 3
    return want * (2 * STEP32 + (adds + 1) * HALF32)
