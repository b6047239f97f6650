"""The mean square that the errors of the 8-bit products may have.

The worst-case bounds of fp8_reference grow with the number of columns, and sums kept in
too few bits fit them.  Errors that are independent add up by their squares.  Here m is
the mean square that one result's error has at most:
  - what the matrix instruction cuts off: of eight neighbouring products each loses what
    it has below 2^(e - 13), e the largest sum of two codes' exponents among them.  The
    loss is known; its sign is the product's, which is random in these tests' data, so
    that the losses' squares add up;
  - 32-bit sums: a whole step of the sum of all magnitudes;
  - one rounding to fp16: evenly spread over a step, a twelfth of its square.
The sum of n squared errors has a standard deviation of at most 1.5 m each (evenly spread
errors 0.9 m, normal ones 1.42 m); `close` allows six of them."""
import numpy as np

import fp8_reference as ref
from fp8_reference import STEP32


class Operand:
    """Rows of codes, as the values that they stand for, with a scale for each 128."""

    def __init__(self, codes, scales):
        self.codes = ref.decoded(codes).astype(np.float32)
        self.scales = np.asarray(scales, np.float64)
        assert self.scales.shape == (self.codes.shape[0], -(-self.codes.shape[1] // 128))
        # exponents; of a code below 2^-6: -6
        self.exponents = (np.frexp(np.maximum(np.abs(self.codes), np.float32(2.0 ** -6)))[1] - 1).astype(np.float32)

    def rows(self, at):
        out = object.__new__(Operand)
        out.codes, out.scales, out.exponents = self.codes[at], self.scales[at], self.exponents[at]
        return out

    @property
    def values(self):
        return self.codes * np.repeat(self.scales, 128, 1)[:, :self.codes.shape[1]]


def activations(x):
    return Operand(*ref.quantize(x))


def matrix(codes, scales, columns=None):
    """A matrix of codes [N][K] and scales [ceil(N/128)][...]; its columns (N) of a sample."""
    columns = np.arange(codes.shape[0]) if columns is None else columns
    return Operand(codes, np.asarray(scales)[columns // 128])


def products(a, w):
    """For each 128 columns: the products [M][N][16][8] (fewer eights at the end) and what
    each loses, exact in 32 bits."""
    for k in range(0, a.codes.shape[1], 128):
        at = slice(k, k + 128)
        p = a.codes[:, None, at] * w.codes[None, :, at]
        p = p.reshape(*p.shape[:2], -1, 8)
        unit = np.exp2((a.exponents[:, None, at] + w.exponents[None, :, at]).reshape(p.shape).max(-1, keepdims=True) - 13)
        yield p, p - np.trunc(p / unit) * unit, a.scales[:, k // 128, None] * w.scales[:, k // 128]


def sum_square(a, w):
    """m of the sums of products of the rows of a and w."""
    m = (STEP32 * (np.abs(a.values) @ np.abs(w.values).T)) ** 2
    step = max(1, (1 << 24) // (w.codes.shape[0] * 128))
    for i in range(0, len(m), step):
        for _, lost, s in products(a.rows(slice(i, i + step)), w):
            m[i:i + step] += (lost ** 2).sum((2, 3), dtype=np.float64) * s ** 2
    return m


def fp16_rounding(y):
    """A twelfth of the square of fp16's step at y."""
    step = np.exp2(np.maximum(np.frexp(np.abs(y))[1] - 11.0, -24.0))
    return step ** 2 / 12


def gemm(x, w, residual=None):
    """The product and m of its results."""
    a = activations(x)
    y, m = a.values @ w.values.T, sum_square(a, w)
    if residual is not None:
        y = y + np.asarray(residual, np.float64)
        m = m + (STEP32 * (np.abs(y) + np.abs(residual).astype(np.float64))) ** 2
    return y, m + fp16_rounding(y)


def swiglu_of(a, wg, wu):
    g, u = a.values @ wg.values.T, a.values @ wu.values.T
    s = 1 / (1 + np.exp(-np.clip(g, -700, 700)))
    h = g * s * u
    # h's slopes by g and by u; the fast exponential and what follows it as in ref.swiglu
    m = (s * (1 + g * (1 - s)) * u) ** 2 * sum_square(a, wg) + (g * s) ** 2 * sum_square(a, wu) + ((4 + np.abs(g)) * STEP32 * h) ** 2
    return h, m + fp16_rounding(h)


def swiglu(x, wg, wu, offsets, rows, k, places):
    """h of some places, and m of its results; wg and wu: an operand for each expert."""
    e_of = ref.expert_of_place(offsets)[places]
    h, m = (np.zeros((len(places), wg[0].codes.shape[0])) for _ in range(2))
    a = activations(x[rows[places] // k])
    for e in np.unique(e_of):
        at = e_of == e
        h[at], m[at] = swiglu_of(a.rows(at), wg[e], wu[e])
    return h, m


def down(h, w, offsets, pos, weights, residual, tokens):
    """y of some tokens, and m of its results."""
    T, k = weights.shape
    e_of = ref.expert_of_place(offsets)
    y = np.zeros((len(tokens), w[0].codes.shape[0])) if residual is None else np.asarray(residual[tokens], np.float64)
    size, m = np.abs(y), np.zeros(y.shape)
    place = pos.reshape(T, k)[tokens]
    for j in range(k):
        for e in range(len(offsets) - 1):
            at = np.flatnonzero(place[:, j] >= 0)
            at = at[e_of[place[at, j]] == e]
            if at.size:
                a, p = activations(h[place[at, j]]), weights[tokens[at], j].astype(np.float64)[:, None]
                o = a.values @ w[e].values.T
                y[at] += p * o
                m[at] += p ** 2 * sum_square(a, w[e])
                size[at] += np.abs(p * o)
    return y, m + (k * STEP32 * size) ** 2 + fp16_rounding(y)


def ratio(got, want, m):
    """The sum of squared errors over what it may be."""
    off = (np.asarray(got, np.float64) - want) ** 2
    return off.sum() / (m.sum() + 6 * 1.5 * np.sqrt((m ** 2).sum()))


def close(got, want, m):
    r = ratio(got.cpu().numpy() if hasattr(got, "cpu") else got, want, m)
    assert r <= 1, r
    return r
