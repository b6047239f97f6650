"""Block-scaled 8-bit matrices on the GPU: quantisation bit for bit, products against
64 bits within the bounds of 32-bit sums and one fp16 rounding."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_mx4 import check, half, strided

pytestmark = pytest.mark.gpu


def quantize(x, rows=1):
    M, K = x.shape
    codes = torch.full((M, K), 0xEE, dtype=torch.uint8, device=dev())
    scales = torch.full((-(-M // rows), -(-K // 128)), 7.0, device=dev())
    ss.fp8_quantize(x, codes, scales, rows=rows)
    return codes, scales


def same(codes, scales, x, rows=1):
    c, s = ref.quantize(x, rows)
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), c)
    return c, s


@pytest.mark.parametrize("M,K,pad", [(1, 16, 0), (3, 64, 8), (17, 144, 0), (5, 160, 40), (2, 4096, 0), (1000, 32, 0), (7, 8208, 16),
                                     (128, 128, 0), (129, 272, 8), (300, 1040, 0)])
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_is_exact(M, K, pad, rows):
    rng = np.random.default_rng(M * K)
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-20, 14, (M, K)))).astype(np.float16)
    codes, scales = quantize(strided(x, pad), rows)
    c, s = same(codes, scales, x, rows)
    out = torch.full((M + 1, K + pad), 7.0, dtype=torch.float16, device=dev())
    ss.fp8_dequantize(codes, scales, out[:M, :K], rows=rows)
    with np.errstate(over="ignore"):
        assert np.array_equal(out[:M, :K].cpu().numpy(), ref.values(c, s, rows).astype(np.float16))
    assert (out[M:] == 7).all() and (out[:, K:] == 7).all()


def test_quantize_every_fp16_value():
    """Each finite value beside a block maximum of each exponent and of the mantissas
    around 1.75: every rounding position, tie and subnormal."""
    bits = np.arange(65536, dtype=np.uint16)
    every = bits[(bits & 0x7C00) != 0x7C00].view(np.float16)
    every = every[np.argsort(np.abs(every.astype(np.float32)), kind="stable")]
    x = every[:every.size // 128 * 128].reshape(-1, 128)
    same(*quantize(half(x)), x)
    for shift in (1, 4, 9):  # each beside a maximum up to 2^9 times as large
        top = np.minimum(np.abs(x).max(-1).astype(np.float64) * 2.0 ** shift * 1.3, 65504).astype(np.float16)
        y = np.concatenate([x, np.repeat(top[:, None], 16, 1)], 1)[:, 16:]
        same(*quantize(half(y)), y)


def test_quantize_largest_of_a_block():
    """The scale's own border: 448 s, and the next value above it."""
    x = np.zeros((60, 128), np.float16)
    for i in range(30):
        top = np.float16(1.75 * 2.0 ** (i - 14))
        x[2 * i, i], x[2 * i + 1, 127 - i] = top, -np.nextafter(top, np.float16(np.inf))
    x[:, 64] = np.float16(2.0 ** -24)
    c, s = same(*quantize(half(x)), x)
    assert (s[1::2] == 2 * s[::2]).all() and (c[::2].max(-1) == 126).all()


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_blocks_without_a_scale(rows):
    x = np.ones((256, 272), np.float16)
    x[0, :128] = 0
    x[0, 5] = -0.0
    x[1, 133] = np.inf
    x[130, 0] = np.nan
    x[255, 271] = -np.inf
    codes, scales = quantize(half(x), rows)
    c, s = same(codes, scales, x, rows)
    y = torch.empty(256, 272, dtype=torch.float16, device=dev())
    ss.fp8_dequantize(codes, scales, y, rows=rows)
    assert np.array_equal(np.isnan(y.cpu().numpy()), np.isnan(np.repeat(np.repeat(s, rows, 0), 128, 1)[:, :272]))


def test_dequantize_every_code():
    codes = np.tile(np.arange(256, dtype=np.uint8), (24, 1))
    scales = np.stack([np.float32(v) * np.float32([1, 1.3]) for v in
                       (*(2.0 ** np.arange(-40, 12, 3)), 0.0, -3.7, 1e30, np.inf, -np.inf, np.nan)]).astype(np.float32)
    y = torch.empty(24, 256, dtype=torch.float16, device=dev())
    ss.fp8_dequantize(up(codes), up(scales), y)
    with np.errstate(over="ignore", invalid="ignore"):
        want = ref.values(codes, scales, rows=1).astype(np.float16)  # the product of 4 and 24 bits is exact in 64
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)


def matrix(rng, *shape):
    c, s = ref.random_matrix(rng, *shape)
    t = up(c), up(s)
    W = ss.make_fp8(*t)
    return W, (t, ss.prepack_fp8(W)), ref.values(c, s)


SIZES = [(1, 16, 16), (1, 2048, 2048), (2, 96, 48), (3, 128, 32), (5, 160, 80), (8, 1040, 112), (13, 4096, 64),
         (15, 512, 16), (16, 656, 96), (17, 2048, 144), (31, 912, 272), (32, 8192, 64), (33, 384, 48), (48, 1424, 128),
         (63, 2064, 64), (64, 4096, 208), (65, 1024, 512), (100, 368, 336), (128, 256, 256), (129, 304, 528),
         (200, 4096, 272), (257, 1168, 304), (300, 14336, 32), (511, 48, 16), (513, 560, 1040),
         (33, 8208, 2080), (40, 28672, 656), (96, 16400, 1056), (130, 14352, 1200), (200, 8192, 2128), (700, 1040, 3600),
         (1030, 14336, 560), (1300, 528, 7056), (2100, 16432, 400), (1800, 16464, 2064),
         (3, 8192, 16400), (11, 4096, 6400), (40, 256, 4112), (100, 144, 2064), (27, 1040, 8208)]


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_gemm(M, K, N, residual):
    rng = np.random.default_rng(M + K + N)
    W, keep, w = matrix(rng, N, K)
    x = rng.standard_normal((M, K)).astype(np.float16)
    x[:, ::37] *= 20
    r = rng.standard_normal((M, N)).astype(np.float16) * 4 if residual else None
    want, bound = ref.gemm(x, w, r)
    out = torch.full((M + 1, N + 12), 7.0, dtype=torch.float16, device=dev())
    y = out[:M, :N]
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N))
    rr = strided(r, 4) if residual else None
    ss.fp8_gemm(W, strided(x, 8), y, ws, residual=rr)
    check(y, want, bound)
    off = np.mean((y.cpu().numpy().astype(np.float64) - want) ** 2)
    if M * N >= 256:  # of few errors the mean square says little
        assert off <= ref.gemm_mean_square(x, w, want), off
    assert (out[M:] == 7).all() and (out[:, N:] == 7).all()
    if residual:  # into the residual stream itself
        s = half(r)
        ss.fp8_gemm(W, half(x), s, ws, residual=s)
        assert torch.equal(s, y)


@pytest.mark.parametrize("M,K,N", [(4, 256, 256), (40, 512, 512), (300, 512, 512)])
def test_gemm_over_its_own_input(M, K, N):
    rng = np.random.default_rng(5)
    W, keep, w = matrix(rng, N, K)
    x = half(rng.standard_normal((M, K)))
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N))
    y = torch.empty(M, N, dtype=torch.float16, device=dev())
    ss.fp8_gemm(W, x, y, ws)
    z = x.clone()
    ss.fp8_gemm(W, z, z, ws)
    assert torch.equal(z, y)


@pytest.mark.parametrize("M,K,N", [(3, 272, 160), (40, 384, 288), (150, 256, 320), (600, 400, 528)])
def test_gemm_extreme_values(M, K, N):
    """Weight scales over the range of a product that fp32 holds, zero and negative ones
    among them, the fp16 extremes as activations, and rows with an infinity or a NaN:
    those are NaN, and no other row is; a NaN among the codes is its column's, a NaN
    among the scales its block's."""
    rng = np.random.default_rng(K)
    c, s = ref.random_matrix(rng, N, K)
    s *= np.exp2(rng.integers(-50, 4, s.shape)).astype(np.float32)
    s[0, 0], s[-1, -1] = 0, -s[-1, -1]
    t = up(c), up(s)
    W = ss.make_fp8(*t)
    packed = ss.prepack_fp8(W)  # noqa: F841
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-24, -1, (M, K)))).astype(np.float16)
    x[0, :] = np.float16(2.0 ** -24)
    x[1, 7], x[2, K - 1] = np.nan, -np.inf
    y = torch.empty(M, N, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N))
    ss.fp8_gemm(W, half(x), y, ws)
    bad = np.zeros(M, bool)
    bad[1:3] = True
    assert np.array_equal(np.isnan(y.cpu().numpy()), np.repeat(bad[:, None], N, 1))
    want, bound = ref.gemm(x[~bad], ref.values(c, s))
    check(y[torch.from_numpy(~bad).to(dev())], want, bound)
    c[N // 2, 1] = 0xFF
    s[1, 1] = np.nan
    t[0].copy_(up(c))
    t[1].copy_(up(s))
    packed = ss.prepack_fp8(W)  # noqa: F841
    ss.fp8_gemm(W, half(x), y, ws)
    n = np.isnan(y.cpu().numpy())[~bad]
    hit = np.zeros(N, bool)
    hit[N // 2] = True
    hit[128:256] = True
    assert np.array_equal(n, np.repeat(hit[None], n.shape[0], 0))


@pytest.mark.parametrize("M,K,N", [(1, 2048, 2048), (32, 2048, 512), (60, 16384, 1152), (400, 1024, 1024)])
def test_gemm_replays_and_repeats(M, K, N):
    """Bit-identical from call to call, with a smaller call on the same workspace
    between, and from a graph."""
    rng = np.random.default_rng(9)
    W, keep, w = matrix(rng, N, K)
    x = half(rng.standard_normal((M, K)))
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N))
    y, z = (torch.empty(M, N, dtype=torch.float16, device=dev()) for _ in range(2))
    ss.fp8_gemm(W, x, y, ws)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        g = ss.Graph()
        g.begin()
        ss.fp8_gemm(W, x, z, ws)
        g.end()
        for _ in range(3):
            z.zero_()
            one = torch.empty(1, N, dtype=torch.float16, device=dev())
            ss.fp8_gemm(W, x[:1], one, ws)
            g.launch()
            st.synchronize()
            assert torch.equal(z, y)
    torch.cuda.current_stream().wait_stream(st)


def test_gemm_uses_the_callers_stream():
    rng = np.random.default_rng(3)
    W, keep, w = matrix(rng, 512, 512)
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(64, 512, 512))
    st = torch.cuda.Stream()
    x = torch.zeros(64, 512, dtype=torch.float16, device=dev())
    y = torch.empty(64, 512, dtype=torch.float16, device=dev())
    v = rng.standard_normal((64, 512)).astype(np.float16)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(1 << 22)
        x.copy_(half(v))
    ss.fp8_gemm(W, x, y, ws, stream=st)
    st.synchronize()
    check(y, *ref.gemm(v, w))


@pytest.mark.parametrize("rows", [1, 128])
def test_the_longest_row(rows):
    """A row of 2^31 - 128 columns, the most."""
    K = 2**31 - 128
    x = torch.zeros(1, K, dtype=torch.float16, device=dev())
    codes, scales = torch.empty(1, K, dtype=torch.uint8, device=dev()), torch.empty(1, 2**24 - 1, device=dev())
    for at, v in ((0, 3.0), (2**30 + 5, 500.0), (K - 1, -900.0)):
        x[0, at] = v
    ss.fp8_quantize(x, codes, scales, rows=rows)
    assert [scales[0, i].item() for i in (0, 1, 2**23, 2**24 - 3, 2**24 - 2)] == [2.0**-7, 1.0, 2.0, 1.0, 4.0]
    assert torch.count_nonzero(codes).item() == 3 and torch.count_nonzero(scales == 1).item() == 2**24 - 4
    y = torch.empty_like(x)
    ss.fp8_dequantize(codes, scales, y, rows=rows)
    assert [y[0, at].item() for at in (0, 2**30 + 5, K - 1)] == [3.0, 512.0, -896.0]
    assert torch.count_nonzero(y).item() == 3


def test_refusals_of_the_binding():
    rng = np.random.default_rng(1)
    W, keep, w = matrix(rng, 64, 128)
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(4, 128, 64))
    x, y = (torch.zeros(4, n, dtype=torch.float16, device=dev()) for n in (128, 64))
    codes, scales = torch.zeros(4, 128, dtype=torch.uint8, device=dev()), torch.zeros(4, 1, device=dev())

    def refused(status, f):
        with pytest.raises(ss.SwiftSpecError) as e:
            f()
        assert e.value.status == status

    bad = ss.INVALID_ARG
    refused(bad, lambda: ss.fp8_gemm(W, x[:, :96], y, ws))             # other K
    refused(bad, lambda: ss.fp8_gemm(W, x, y[:, :32], ws))             # other N
    refused(bad, lambda: ss.fp8_gemm(W, x, y[:3], ws))                 # other M
    refused(bad, lambda: ss.fp8_gemm(W, x.float(), y, ws))             # other type
    refused(bad, lambda: ss.fp8_gemm(W, torch.zeros(128, 4, dtype=torch.float16, device=dev()).T, y, ws))
    refused(bad, lambda: ss.fp8_gemm(W, x.cpu(), y, ws))               # not on the GPU
    refused(bad, lambda: ss.fp8_gemm(W, x, y, ws, residual=y[:2]))
    refused(ss.WORKSPACE_TOO_SMALL, lambda: ss.fp8_gemm(W, x, y, ws[:1024]))
    refused(ss.MISALIGNED, lambda: ss.fp8_gemm(W, torch.zeros(4, 132, dtype=torch.float16, device=dev())[:, :128], y, ws))
    refused(bad, lambda: ss.fp8_quantize(x, codes, scales[:3]))
    refused(bad, lambda: ss.fp8_quantize(x, codes, scales, rows=2))
    refused(bad, lambda: ss.fp8_quantize(x, codes, scales, rows=128))  # one row of scales
    refused(bad, lambda: ss.fp8_quantize(x, codes[:, :64], scales))
    refused(bad, lambda: ss.fp8_dequantize(codes, scales.to(torch.int32), x))
    refused(ss.MISALIGNED, lambda: ss.fp8_quantize(x, torch.zeros(516, dtype=torch.uint8, device=dev())[4:].view(4, 128), scales))
    refused(bad, lambda: ss.make_fp8(keep[0][0], keep[0][1][:0]))
    refused(bad, lambda: ss.make_fp8(keep[0][0].view(torch.float8_e5m2), keep[0][1]))
    refused(bad, lambda: ss.make_fp8(*keep[0], packed=keep[1][:64]))
    typed = ss.make_fp8(keep[0][0].view(torch.float8_e4m3fn), keep[0][1], packed=keep[1])
    z = torch.ones_like(y)
    ss.fp8_gemm(typed, x, z, ws)
    assert (z == 0).all()
    ss.fp8_gemm(W, x[:0], y[:0], ws)  # no rows: nothing to do
