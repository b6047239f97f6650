"""CPU checks of the block-scaled 8-bit entry points and of the router with scores:
sizes, and bad arguments rejected on the host before any launch; and the host
reference of their GPU tests against closed forms."""
import ctypes

import numpy as np
import pytest

import fp8_reference as ref
from test_abi import ss  # noqa: F401  (fixture: the built library)
from test_mx4_abi import BIG, FAKE, bad_groups, groups, status


def test_sizes(ss):  # noqa: F811
    lib = ss.lib()
    # 16 x 128 blocks of 2 KB, a float for 128 x 128 values
    assert lib.swiftspec_fp8_packed_bytes(128, 16, 1) == 2048 + 4
    assert lib.swiftspec_fp8_packed_bytes(512, 16, 3) == 3 * (4 * 2048 + 4 * 4)
    assert lib.swiftspec_fp8_packed_bytes(528, 144, 1) == 9 * 5 * 2048 + 2 * 5 * 4
    assert lib.swiftspec_fp8_packed_bytes(0, 16, 1) == 0
    assert lib.swiftspec_fp8_packed_bytes(65536, 65536, 1) == 0  # 4 GiB
    for f, a in (("fp8_gemm", (0, 128, 16)), ("moe_fp8_swiglu", (0, 2, 4, 128, 16)), ("moe_fp8_down", (0, 2, 4, 128, 16))):
        assert getattr(lib, f"swiftspec_{f}_workspace_bytes")(*a) == ss.WS_HEADER_BYTES
    # the query of the most rows serves every smaller number
    for K, N in ((4096, 4096), (28672, 8192), (14336, 512), (16400, 16)):
        sizes = [lib.swiftspec_fp8_gemm_workspace_bytes(m, K, N) for m in range(3000)]
        assert sizes == sorted(sizes)
    for f in ("swiglu", "down"):
        q = getattr(lib, f"swiftspec_moe_fp8_{f}_workspace_bytes")
        assert all(q(t, 4, 32, 512, 256) <= q(300, 4, 32, 512, 256) for t in range(300))
    assert ss.fp8_gemm_workspace_bytes(1 << 40, 128, 16) == ss.WS_HEADER_BYTES


def test_matrix_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = lambda K=128, N=64, E=1, packed=FAKE, codes=FAKE, scales=FAKE: ss.FP8(codes, scales, K, N, E, packed)  # noqa: E731
    pack = lambda w, out=FAKE, size=BIG: status(lib, "fp8_prepack", ctypes.byref(w), out, size)  # noqa: E731
    assert status(lib, "fp8_prepack", None, FAKE, BIG) == ss.INVALID_ARG
    assert pack(W(K=0)) == pack(W(N=0)) == pack(W(E=0)) == pack(W(codes=None)) == pack(W(scales=None)) == pack(W(), out=None) == ss.INVALID_ARG
    assert pack(W(K=40)) == pack(W(N=24)) == pack(W(E=513)) == ss.UNSUPPORTED
    assert pack(W(K=65536, N=65536)) == ss.UNSUPPORTED       # 4 GiB and more
    assert pack(W(K=32768, N=4096, E=256)) == ss.UNSUPPORTED  # all of them 32 GiB and more
    assert pack(W(codes=FAKE + 8)) == pack(W(), out=FAKE + 4) == pack(W(scales=FAKE + 2)) == ss.MISALIGNED
    assert pack(W(), size=lib.swiftspec_fp8_packed_bytes(128, 64, 1) - 1) == ss.WORKSPACE_TOO_SMALL
    quant = lambda x=FAKE, M=4, K=64, ld=64, b=1, c=FAKE, s=FAKE: status(lib, "fp8_quantize", x, M, K, ld, b, c, s)  # noqa: E731
    back = lambda x=FAKE, M=4, K=64, ld=64, b=1, c=FAKE, s=FAKE: status(lib, "fp8_dequantize", c, s, M, K, b, x, ld)  # noqa: E731
    for f in (quant, back):
        assert f(x=None) == f(c=None) == f(s=None) == f(M=-1) == f(K=0) == f(ld=32) == f(b=0) == f(b=64) == ss.INVALID_ARG
        assert f(K=40) == f(M=1 << 50) == f(M=(1 << 35) // 128) == ss.UNSUPPORTED
        for b in (1, 128):  # 2^31 columns and more, rounded up to whole blocks
            assert f(M=1, K=(1 << 31) - 16, ld=1 << 31, b=b) == f(M=1, K=(1 << 31) - 112, ld=1 << 31, b=b) == ss.UNSUPPORTED
        assert f(x=FAKE + 2) == f(ld=68) == f(c=FAKE + 4) == f(s=FAKE + 2) == ss.MISALIGNED
        assert f(M=0) == f(M=0, b=128) == ss.OK


def test_gemm_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = ss.FP8(FAKE, FAKE, 128, 64, 1, FAKE)

    def gemm(w=W, x=FAKE, M=4, ldx=128, y=FAKE, ldy=64, r=None, ldr=0, ws=FAKE, size=BIG):
        return status(lib, "fp8_gemm", ctypes.byref(w) if w else None, x, M, ldx, y, ldy, r, ldr, ws, size)

    assert gemm(w=None) == gemm(x=None) == gemm(y=None) == gemm(ws=None) == ss.INVALID_ARG
    assert gemm(w=ss.FP8(FAKE, FAKE, 128, 64, 1, None)) == gemm(w=ss.FP8(FAKE, FAKE, 128, 64, 2, FAKE)) == ss.INVALID_ARG
    assert gemm(M=-1) == gemm(ldx=120) == gemm(ldy=60) == gemm(r=FAKE + 64, ldr=60) == ss.INVALID_ARG
    assert gemm(r=FAKE, ldr=128) == ss.INVALID_ARG  # over y with another row length
    assert gemm(M=1 << 24) == ss.UNSUPPORTED        # 2 GiB of rows
    assert gemm(x=FAKE + 2) == gemm(ldx=132) == gemm(y=FAKE + 4) == gemm(ldy=66) == gemm(ws=FAKE + 8) == ss.MISALIGNED
    assert gemm(r=FAKE + 4, ldr=64) == gemm(r=FAKE + 64, ldr=66) == gemm(w=ss.FP8(FAKE, FAKE, 128, 64, 1, FAKE + 8)) == ss.MISALIGNED
    assert gemm(size=lib.swiftspec_fp8_gemm_workspace_bytes(4, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL
    assert gemm(M=0) == ss.OK


def test_experts_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = lambda K=128, N=64, E=8, packed=FAKE: ctypes.byref(ss.FP8(FAKE, FAKE, K, N, E, packed))  # noqa: E731

    def swiglu(w=W(), u=W(), x=FAKE, ldx=128, g=groups(ss), h=FAKE, ldh=64, ws=FAKE, size=BIG):
        return status(lib, "moe_fp8_swiglu", w, u, x, ldx, g, h, ldh, ws, size)

    def down(w=W(), h=FAKE, ldh=128, g=groups(ss), p=FAKE, y=FAKE, ldy=64, r=None, ldr=0, ws=FAKE, size=BIG):
        return status(lib, "moe_fp8_down", w, h, ldh, g, p, y, ldy, r, ldr, ws, size)

    for want, g in bad_groups(ss):
        assert swiglu(g=g) == down(g=g) == want
    for f in (swiglu, down):
        assert f(w=None) == f(h=None) == f(ws=None) == f(ldh=56) == f(w=W(packed=None)) == f(w=W(E=7)) == ss.INVALID_ARG
        assert f(h=FAKE + 2) == f(ldh=130) == f(ws=FAKE + 8) == ss.MISALIGNED
        assert f(g=groups(ss, T=0)) == ss.OK
    assert swiglu(x=None) == swiglu(u=None) == swiglu(u=W(K=256)) == swiglu(u=W(N=32)) == swiglu(ldx=120) == ss.INVALID_ARG
    assert swiglu(g=groups(ss, T=1 << 25, k=1)) == down(g=groups(ss, T=1 << 25, k=1)) == ss.UNSUPPORTED
    assert swiglu(x=FAKE + 2) == swiglu(ldx=132) == ss.MISALIGNED
    assert down(p=None) == down(y=None) == down(ldy=60) == down(r=FAKE, ldr=128) == down(r=FAKE + 64, ldr=60) == ss.INVALID_ARG
    assert down(y=FAKE + 4) == down(ldy=66) == down(p=FAKE + 2) == down(r=FAKE + 4, ldr=64) == down(r=FAKE + 64, ldr=66) == ss.MISALIGNED
    assert swiglu(size=lib.swiftspec_moe_fp8_swiglu_workspace_bytes(4, 2, 8, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL
    assert down(size=lib.swiftspec_moe_fp8_down_workspace_bytes(4, 2, 8, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL


def test_launches_of_too_many_threads(ss):  # noqa: F811
    lib = ss.lib()
    W = lambda K, N, E: ctypes.byref(ss.FP8(FAKE, FAKE, K, N, E, FAKE))  # noqa: E731
    G = lambda T, k, E: groups(ss, T=T, k=k, E=E)  # noqa: E731
    # 4000 pairs of 512 experts over 2 x 393216 columns: up to 762 blocks of 16 rows
    wide = W(128, 393216, 512)
    assert status(lib, "moe_fp8_swiglu", wide, wide, FAKE, 128, G(250, 16, 512), FAKE, 393216, FAKE, BIG) == ss.UNSUPPORTED
    # four results a thread of the combination
    assert status(lib, "moe_fp8_down", W(128, 8192, 8), FAKE, 128, G(1 << 20, 1, 8), FAKE, FAKE, 8192, None, 0, FAKE, BIG) == ss.UNSUPPORTED


def test_route_refusals(ss):  # noqa: F811
    lib = ss.lib()

    def route(g=groups(ss), x=FAKE, bits=32, ld=8, e=FAKE, w=FAKE, ws=FAKE, size=BIG, null=False, **how):
        s = dict(score=1, groups=4, top_groups=2, group_best=2, renormalize=1, scale=1.0, bias=FAKE)
        s.update(how)
        return status(lib, "moe_route_scored", x, bits, ld, None if null else ctypes.byref(ss._Scoring(**s)), e, w, g, ws, size)

    for want, g in bad_groups(ss):
        assert route(g=g) == want
    assert route(x=None) == route(e=None) == route(w=None) == route(ws=None) == route(ld=7) == route(null=True) == ss.INVALID_ARG
    assert route(bits=64) == route(bits=0) == route(score=2) == route(score=-1) == route(group_best=0) == route(group_best=3) == ss.INVALID_ARG
    assert route(groups=0) == route(groups=3) == route(groups=16) == route(top_groups=0) == route(top_groups=5) == ss.INVALID_ARG
    assert route(x=FAKE + 1, bits=16) == route(x=FAKE + 2) == route(e=FAKE + 2) == route(w=FAKE + 2) == route(bias=FAKE + 2) == ss.MISALIGNED
    assert route(ws=FAKE + 4) == ss.MISALIGNED
    assert route(size=lib.swiftspec_moe_route_workspace_bytes(4, 8, 2) - 1) == ss.WORKSPACE_TOO_SMALL


def test_tensors_that_the_library_would_read_differently(ss):  # noqa: F811
    torch = pytest.importorskip("torch")

    def refused(f, *args, **named):
        with pytest.raises(ss.SwiftSpecError) as e:
            f(*args, **named)
        assert e.value.status == ss.INVALID_ARG

    codes, scales = torch.zeros(144, 160, dtype=torch.uint8), torch.zeros(2, 2)
    refused(ss.make_fp8, codes, scales)  # not on a GPU
    meta = lambda t: t.to("meta")  # noqa: E731
    for c, s in ((codes, scales[:1]), (codes, scales.double()), (codes, torch.zeros(2, 2, dtype=torch.int32)), (codes.T, scales),
                 (codes.to(torch.int16), scales), (codes.view(torch.float8_e5m2), scales), (codes.view(torch.float8_e4m3fnuz), scales)):
        refused(ss.make_fp8, meta(c), meta(s))
    assert ss._rows(torch.empty(3, 8, device="meta"), "", 8, dtype=torch.float32) == (3, 8)
    refused(ss._rows, torch.empty(3, 8, device="meta"), "", 8)


def test_reference_quantization():
    # codes of a block whose scale is 1, and ties between them
    x = np.zeros((1, 128), np.float16)
    x[0, :16] = [448, 232, 248, -248, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10, 1.0625, 1.1875, -1.0, 0.0156, 300, 432, 0.5, -6]
    codes, scales = ref.quantize(x)
    assert scales.tolist() == [[1]]
    assert ref.values(codes, scales, 1)[0, :16].tolist() == [448, 224, 256, -256, 2.0 ** -9, 0, 2.0 ** -8, 2.0 ** -8, 1, 1.25, -1, 0.015625,
                                                             288, 448, 0.5, -6]
    # homogeneous under powers of two, and at most half a step off
    rng = np.random.default_rng(0)
    v = rng.standard_normal((5, 272)).astype(np.float16)
    q = ref.quantized(v)
    assert np.array_equal(ref.quantized(v * np.float16(0.25)), q / 4)
    s = np.repeat(ref.quantize(v)[1], 128, 1)[:, :272]
    assert (np.abs(q - v) <= np.maximum(np.abs(v.astype(np.float64)) / 16, s * 2.0 ** -10)).all()
    whole = ref.quantize(v, 128)[1]
    assert whole.shape == (1, 3) and np.array_equal(whole[0], ref.quantize(v)[1].max(0))


def test_reference_scores():
    """Gates, groups and bias where they can be worked out by hand."""
    x = np.float32([[0, 1, 2, 3, 4, 5, -1, -2]])
    sig = 1 / (1 + np.exp(-x[0].astype(np.float64)))
    e, w = ref.route(x, 2, "sigmoid", renormalize=False)
    assert e.tolist() == [[5, 4]] and np.allclose(w, sig[[5, 4]])
    # pairs as groups: the best is {4, 5}; with a bias on 0 and 6 the sums change, the weights do not
    e, w = ref.route(x, 2, "sigmoid", groups=4, top_groups=1, group_best=2)
    assert e.tolist() == [[5, 4]] and np.allclose(w.sum(), 1)
    b = np.float32([3, 0, 0, 0, 0, 0, 2, 0])
    e, w = ref.route(x, 3, "sigmoid", b, groups=4, top_groups=2, group_best=1, renormalize=False, scale=2)
    assert e.tolist() == [[0, 6, 1]] and np.allclose(w, 2 * sig[[0, 6, 1]])
    e, w = ref.route(x, 3, "softmax", groups=4, top_groups=1)  # one slot stays empty
    p = np.exp(x[0].astype(np.float64))
    assert e.tolist() == [[5, 4, -1]] and np.allclose(w, [[p[5] / (p[4] + p[5]), p[4] / (p[4] + p[5]), 0]])
    plain, _ = ref.route(x, 3, "softmax", renormalize=False)
    assert plain.tolist() == [[5, 4, 3]]
    e, w = ref.route(np.full((1, 8), -np.inf, np.float32), 2, "sigmoid")
    assert e.tolist() == [[-1, -1]] and w.tolist() == [[0, 0]]


def test_reference_block_of_one_expert_is_a_dense_one():
    rng = np.random.default_rng(1)
    T, H, F = 6, 144, 48
    x = rng.standard_normal((T, H)).astype(np.float16)
    wg, wu, wd = (ref.values(*ref.random_matrix(rng, 1, *s)) for s in ((F, H), (F, H), (H, F)))
    offsets, rows, pos = ref.group(np.zeros((T, 1), np.int32), 1)
    h, _ = ref.swiglu(x, wg, wu, offsets, rows, 1)
    g, u = ref.quantized(x) @ wg[0].T, ref.quantized(x) @ wu[0].T
    assert np.allclose(h, g / (1 + np.exp(-g)) * u)
    h16 = h.astype(np.float16)
    y, _ = ref.down(h16, wd, offsets, pos, np.ones((T, 1), np.float32))
    assert np.allclose(y, ref.gemm(h16, wd[0])[0])
