"""CPU checks of the bound on the mean square of the 8-bit products' errors: it holds for
what the kernels do, and for nothing that keeps fewer bits."""
import numpy as np
import pytest

import fp8_precision as prec
import fp8_reference as ref


def bf16(v):
    b = np.asarray(v, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + (b >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def fp16(v):
    return np.asarray(v).astype(np.float16).astype(np.float64)


def sums(x, w, scale_of=lambda s: s, part=lambda v: v):
    """[M][N] as the matrix instruction makes them; scale_of: what becomes of the matrix's
    scales, part: of the running sum after each 128 columns."""
    a, w = prec.activations(x), prec.matrix(*w)
    w.scales = scale_of(w.scales)
    y = 0.0
    for p, lost, s in prec.products(a, w):
        y = part(y + (p - lost).sum((2, 3), dtype=np.float64) * s)
    return y


@pytest.fixture(params=[272, 1184])
def data(request):
    """x [96][K] and three matrices of 96 columns, as the GPU tests draw them: over 9000
    results, six standard deviations of whose mean square are a tenth to a fifth of it."""
    K = request.param
    rng = np.random.default_rng(K)
    x = rng.standard_normal((96, K)).astype(np.float16)
    return x, [ref.random_matrix(rng, 96, K) for _ in range(3)], rng


def test_gemm(data):
    x, (w, _, _), rng = data
    want, m = prec.gemm(x, prec.matrix(*w))
    good = sums(x, w)
    prec.close(fp16(good), want, m)
    r = rng.standard_normal(want.shape).astype(np.float16) * 4
    prec.close(fp16(good + r), *prec.gemm(x, prec.matrix(*w), r))
    half = x.shape[1] // 256 * 128
    for name, got in (("running sum in fp16", sums(x, w, part=fp16)), ("scales in bf16", sums(x, w, scale_of=bf16)), ("result in bf16", bf16(good)),
                      ("shares of K in fp16", fp16(sums(x[:, :half], (w[0][:, :half], w[1][:, :half // 128]))) +
                       fp16(sums(x[:, half:], (w[0][:, half:], w[1][:, half // 128:])))),
                      ("activations of fewer bits", sums(fp16(bf16(x)).astype(np.float16), w))):
        assert prec.ratio(fp16(got), want, m) > 1, name


def test_swiglu(data):
    x, (wg, wu, _), _ = data
    offsets, rows, _ = ref.group(np.zeros((96, 1), np.int32), 1)
    want, m = prec.swiglu(x, [prec.matrix(*wg)], [prec.matrix(*wu)], offsets, rows, 1, np.arange(96))
    silu = lambda g, u: g / (1 + np.exp(-g)) * u  # noqa: E731
    g, u = sums(x, wg), sums(x, wu)
    prec.close(fp16(silu(g, u)), want, m)
    for name, got in (("gate and up in fp16", silu(fp16(g), fp16(u))), ("scales in bf16", silu(sums(x, wg, scale_of=bf16), sums(x, wu, scale_of=bf16))),
                      ("running sums in fp16", silu(sums(x, wg, part=fp16), sums(x, wu, part=fp16))), ("result in bf16", bf16(silu(g, u)))):
        assert prec.ratio(fp16(got), want, m) > 1, name


def test_down(data):
    h, ws, rng = data
    k, T = 2, 48
    experts = np.stack([rng.permutation(3)[:k] for _ in range(T)]).astype(np.int32)
    experts[3] = -1
    offsets, rows, pos = ref.group(experts, 3)
    p = rng.random((T, k)).astype(np.float32)
    full = [prec.matrix(*w) for w in ws]
    r = rng.standard_normal((T, 96)).astype(np.float16)
    tokens = np.arange(T)
    place = pos.reshape(T, k)

    def made(row=lambda v: v, **how):
        y = r.astype(np.float64)
        for e in range(3):
            o = row(sums(h, ws[e], **how))
            for t, j in np.argwhere(experts == e):
                y[t] += p[t, j].astype(np.float64) * o[place[t, j]]
        return y

    want, m = prec.down(h, full, offsets, pos, p, r, tokens)
    good = made()
    prec.close(fp16(good), want, m)
    for name, got in (("experts' rows in fp16", made(fp16)), ("scales in bf16", made(scale_of=bf16)), ("running sums in fp16", made(part=fp16)),
                      ("result in bf16", bf16(good))):
        assert prec.ratio(fp16(got), want, m) > 1, name
