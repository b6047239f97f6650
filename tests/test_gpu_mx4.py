"""Microscaled 4-bit matrices on the GPU: quantisation bit for bit, products
against 64 bits within the bounds of 32-bit sums and one fp16 rounding."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up

pytestmark = pytest.mark.gpu


def half(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float16)).to(dev())


def strided(a, pad):
    """The rows of a in a buffer `pad` columns wider, with NaN behind each."""
    t = torch.full((a.shape[0], a.shape[1] + pad), float("nan"), dtype=torch.float16, device=dev())
    t[:, :a.shape[1]] = half(a)
    return t[:, :a.shape[1]]


def quantize(x):
    M, K = x.shape
    codes = torch.full((M, K // 2), 0xEE, dtype=torch.uint8, device=dev())
    scales = torch.full((M, K // 32), 0xEE, dtype=torch.uint8, device=dev())
    ss.mx4_quantize(x, codes, scales)
    return codes, scales


def check(y, want, bound):
    got = y.cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {want[bad][0]} +- {bound[bad][0]}")


@pytest.mark.parametrize("M,K,pad", [(1, 32, 0), (3, 64, 8), (17, 96, 0), (5, 160, 40), (2, 4096, 0), (1000, 32, 0), (7, 8224, 16)])
def test_quantize_is_exact(M, K, pad):
    rng = np.random.default_rng(M * K)
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-20, 14, (M, K)))).astype(np.float16)
    codes, scales = quantize(strided(x, pad))
    c, s = ref.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), c)
    y = torch.empty(M, K + pad, dtype=torch.float16, device=dev())[:, :K]
    ss.mx4_dequantize(codes, scales, y)
    assert np.array_equal(y.cpu().numpy(), ref.values(c, s).astype(np.float16))


def test_quantize_every_fp16_value():
    """Each finite value beside a block maximum of each exponent: every rounding
    position, tie and subnormal."""
    bits = np.arange(65536, dtype=np.uint16)
    every = bits[(bits & 0x7C00) != 0x7C00].view(np.float16)
    every = every[np.argsort(np.abs(every.astype(np.float32)), kind="stable")]
    x = every[:every.size // 32 * 32].reshape(-1, 32)
    codes, scales = quantize(half(x))
    c, s = ref.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), s) and np.array_equal(codes.cpu().numpy(), c)


def test_quantize_blocks_without_a_scale():
    x = np.ones((4, 64), np.float16)
    x[0, :32] = 0
    x[0, 5] = -0.0
    x[1, 33] = np.inf
    x[2, 0] = np.nan
    x[3, 63] = -np.inf
    codes, scales = quantize(half(x))
    c, s = ref.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), s) and np.array_equal(codes.cpu().numpy(), c)
    assert s.tolist() == [[127, 125], [125, 255], [255, 125], [125, 255]]
    y = torch.empty(4, 64, dtype=torch.float16, device=dev())
    ss.mx4_dequantize(codes, scales, y)
    assert np.array_equal(np.isnan(y.cpu().numpy()), np.repeat(s == 255, 32, -1))


def test_dequantize_every_code_and_scale():
    codes = np.tile(np.arange(16, dtype=np.uint8) * 17, (256, 1))  # 16 bytes: each code twice
    scales = np.arange(256, dtype=np.uint8)[:, None]
    y = torch.empty(256, 32, dtype=torch.float16, device=dev())
    ss.mx4_dequantize(up(codes), up(scales), y)
    with np.errstate(over="ignore"):
        want = ref.values(codes, scales).astype(np.float16)
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)


def matrix(rng, *shape, **kw):
    c, s = ref.random_matrix(rng, *shape, **kw)
    t = up(c), up(s)
    W = ss.make_mx4(*t)
    return W, (t, ss.prepack_mx4(W)), ref.values(c, s)


SIZES = [(1, 32, 16), (1, 2048, 2048), (2, 96, 48), (3, 128, 32), (5, 160, 80), (8, 1056, 112), (13, 4096, 64),
         (15, 512, 16), (16, 640, 96), (17, 2048, 144), (31, 896, 272), (32, 8192, 64), (33, 384, 48), (48, 1408, 128),
         (63, 2080, 64), (64, 4096, 208), (65, 1024, 512), (100, 352, 336), (128, 256, 256), (129, 288, 528),
         (200, 4096, 272), (257, 1152, 304), (300, 14336, 32), (511, 64, 16), (513, 544, 1040),
         # few rows over much to read, K split between workgroups, tiles of 128 and 256 rows
         (33, 8224, 2080), (40, 28672, 656), (96, 16416, 1056), (130, 14368, 1200), (200, 8192, 2128), (700, 1056, 3600),
         (1030, 14336, 560), (1300, 544, 7056), (2100, 16448, 400), (1800, 16448, 2064),
         # 16 and 32 rows a workgroup
         (3, 8192, 16400), (11, 4096, 6400), (40, 256, 4112), (100, 160, 2064), (27, 1056, 8208)]


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
    ws = ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N))
    rr = strided(r, 4) if residual else None
    ss.mx4_gemm(W, strided(x, 8), y, ws, residual=rr)
    check(y, want, bound)
    assert (out[M:] == 7).all() and (out[:, N:] == 7).all()
    if residual:  # into the residual stream itself
        s = half(r)
        ss.mx4_gemm(W, half(x), s, ws, residual=s)
        assert torch.equal(s, y)


@pytest.mark.parametrize("M,K,N", [(4, 256, 256), (40, 512, 512), (300, 512, 512)])
def test_gemm_over_its_own_input(M, K, N):
    rng = np.random.default_rng(5)
    W, keep, w = matrix(rng, N, K)
    x = half(rng.standard_normal((M, K)))
    ws = ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N))
    y = torch.empty(M, N, dtype=torch.float16, device=dev())
    ss.mx4_gemm(W, x, y, ws)
    z = x.clone()
    ss.mx4_gemm(W, z, z, ws)
    assert torch.equal(z, y)


@pytest.mark.parametrize("M,K,N", [(3, 256, 64), (40, 384, 96), (150, 256, 320)])
def test_gemm_extreme_scales_and_rows_without_a_value(M, K, N):
    """Weight scales over the whole range of a product that fp32 holds, the fp16
    extremes as activations, and rows with an infinity or a NaN: those are NaN,
    and no other row is."""
    rng = np.random.default_rng(K)
    c, s = ref.random_matrix(rng, N, K)
    s[:] = rng.integers(60, 128, s.shape)
    t = up(c), up(s)
    W = ss.make_mx4(*t)
    packed = ss.prepack_mx4(W)  # noqa: F841
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-24, -1, (M, K)))).astype(np.float16)
    x[0, :] = np.float16(2.0 ** -24)
    x[1, 7], x[2, K - 1] = np.nan, -np.inf
    y = torch.empty(M, N, dtype=torch.float16, device=dev())
    ss.mx4_gemm(W, half(x), y, ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N)))
    bad = np.zeros(M, bool)
    bad[1:3] = True
    assert np.array_equal(np.isnan(y.cpu().numpy()), np.repeat(bad[:, None], N, 1))
    want, bound = ref.gemm(x[~bad], ref.values(c, s))
    check(y[torch.from_numpy(~bad).to(dev())], want, bound)
    # a weight block without a scale: its column, and no other
    s[N // 2, 1] = 255
    t[1].copy_(up(s))
    packed = ss.prepack_mx4(W)  # noqa: F841
    ss.mx4_gemm(W, half(x), y, ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N)))
    n = np.isnan(y.cpu().numpy())[~bad]
    assert n[:, N // 2].all() and n.sum() == n.shape[0]


@pytest.mark.parametrize("M,K,N", [(1, 2048, 2048), (32, 2048, 512), (60, 16384, 1152), (400, 1024, 1024)])
def test_gemm_replays_and_repeats(M, K, N):
    """Bit-identical from call to call, with a smaller call on the same
    workspace between, and from a graph."""
    rng = np.random.default_rng(9)
    W, keep, w = matrix(rng, N, K)
    x = half(rng.standard_normal((M, K)))
    ws = ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N))
    y, z = (torch.empty(M, N, dtype=torch.float16, device=dev()) for _ in range(2))
    ss.mx4_gemm(W, x, y, ws)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        g = ss.Graph()
        g.begin()
        ss.mx4_gemm(W, x, z, ws)
        g.end()
        for _ in range(3):
            z.zero_()
            one = torch.empty(1, N, dtype=torch.float16, device=dev())
            ss.mx4_gemm(W, x[:1], one, ws)
            g.launch()
            st.synchronize()
            assert torch.equal(z, y)
    torch.cuda.current_stream().wait_stream(st)


def test_gemm_uses_the_callers_stream():
    rng = np.random.default_rng(3)
    W, keep, w = matrix(rng, 512, 512)
    ws = ss.workspace(ss.mx4_gemm_workspace_bytes(64, 512, 512))
    st = torch.cuda.Stream()
    x = torch.zeros(64, 512, dtype=torch.float16, device=dev())
    y = torch.empty(64, 512, dtype=torch.float16, device=dev())
    v = rng.standard_normal((64, 512)).astype(np.float16)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(1 << 22)
        x.copy_(half(v))
    ss.mx4_gemm(W, x, y, ws, stream=st)
    st.synchronize()
    check(y, *ref.gemm(v, w))


def test_refusals_of_the_binding():
    rng = np.random.default_rng(1)
    W, keep, w = matrix(rng, 64, 128)
    ws = ss.workspace(ss.mx4_gemm_workspace_bytes(4, 128, 64))
    x, y = (torch.zeros(4, n, dtype=torch.float16, device=dev()) for n in (128, 64))

    def refused(status, f):
        with pytest.raises(ss.SwiftSpecError) as e:
            f()
        assert e.value.status == status

    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x[:, :96], y, ws))             # other K
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x, y[:, :32], ws))             # other N
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x, y[:3], ws))                 # other M
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x.float(), y, ws))             # other type
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, torch.zeros(128, 4, dtype=torch.float16, device=dev()).T, y, ws))
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x.cpu(), y, ws))               # not on the GPU
    refused(ss.INVALID_ARG, lambda: ss.mx4_gemm(W, x, y, ws, residual=y[:2]))
    refused(ss.WORKSPACE_TOO_SMALL, lambda: ss.mx4_gemm(W, x, y, ws[:1024]))
    refused(ss.MISALIGNED, lambda: ss.mx4_gemm(W, torch.zeros(4, 132, dtype=torch.float16, device=dev())[:, :128], y, ws))
    refused(ss.INVALID_ARG, lambda: ss.mx4_quantize(x, keep[0][0], keep[0][1]))
    refused(ss.INVALID_ARG, lambda: ss.make_mx4(keep[0][0], keep[0][1][:, :2]))
    ss.mx4_gemm(W, x[:0], y[:0], ws)  # no rows: nothing to do
