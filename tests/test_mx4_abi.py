"""CPU checks of the microscaled 4-bit and mixture entry points: sizes, and bad
arguments rejected on the host before any launch; and the host reference of
their GPU tests against closed forms."""
import ctypes

import numpy as np
import pytest

import mx4_reference as ref
from test_abi import ss  # noqa: F401  (fixture: the built library)

FAKE = 0x10000  # never dereferenced: validation fails first
BIG = 1 << 40


def status(lib, name, *args):
    return getattr(lib, "swiftspec_" + name)(*args, None)


def test_sizes(ss):  # noqa: F811
    lib = ss.lib()
    # 16 x 128 blocks of 1 KB and a scale word for four of them
    assert lib.swiftspec_mx4_packed_bytes(128, 16, 1) == 1024 + 256
    assert lib.swiftspec_mx4_packed_bytes(512, 16, 3) == 3 * (4096 + 256)
    assert lib.swiftspec_mx4_packed_bytes(544, 32, 1) == 2 * (5 * 1024 + 2 * 256)
    assert lib.swiftspec_mx4_packed_bytes(0, 16, 1) == 0
    for f, a in (("mx4_gemm", (0, 128, 16)), ("moe_route", (0, 4, 2)), ("moe_mx4_swiglu", (0, 2, 4, 128, 16)),
                 ("moe_mx4_down", (0, 2, 4, 128, 16))):
        assert getattr(lib, f"swiftspec_{f}_workspace_bytes")(*a) == ss.WS_HEADER_BYTES
    # the query of the most rows serves every smaller number
    for K, N in ((4096, 4096), (28672, 8192), (14336, 512), (16416, 16)):
        sizes = [lib.swiftspec_mx4_gemm_workspace_bytes(m, K, N) for m in range(3000)]
        assert sizes == sorted(sizes)
    for f in ("swiglu", "down"):
        q = getattr(lib, f"swiftspec_moe_mx4_{f}_workspace_bytes")
        assert all(q(t, 4, 32, 512, 256) <= q(300, 4, 32, 512, 256) for t in range(300))
    assert all(lib.swiftspec_moe_route_workspace_bytes(t, 64, 8) <= lib.swiftspec_moe_route_workspace_bytes(t + 1, 64, 8)
               for t in range(1, 40000, 7))


def test_matrix_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = lambda K=128, N=64, E=1, packed=FAKE, codes=FAKE: ss.MX4(codes, FAKE, K, N, E, packed)  # noqa: E731
    pack = lambda w, out=FAKE, size=BIG: status(lib, "mx4_prepack", ctypes.byref(w), out, size)  # noqa: E731
    assert status(lib, "mx4_prepack", None, FAKE, BIG) == ss.INVALID_ARG
    assert pack(W(K=0)) == pack(W(N=0)) == pack(W(E=0)) == pack(W(codes=None)) == pack(W(), out=None) == ss.INVALID_ARG
    assert pack(W(K=48)) == pack(W(N=24)) == pack(W(E=513)) == ss.UNSUPPORTED
    assert pack(W(K=131072, N=131072)) == ss.UNSUPPORTED  # 4 GiB and more
    assert pack(W(codes=FAKE + 8)) == pack(W(), out=FAKE + 4) == ss.MISALIGNED
    assert pack(W(), size=lib.swiftspec_mx4_packed_bytes(128, 64, 1) - 1) == ss.WORKSPACE_TOO_SMALL
    quant = lambda x=FAKE, M=4, K=64, ld=64, c=FAKE, s=FAKE: status(lib, "mx4_quantize", x, M, K, ld, c, s)  # noqa: E731
    back = lambda x=FAKE, M=4, K=64, ld=64, c=FAKE, s=FAKE: status(lib, "mx4_dequantize", c, s, M, K, x, ld)  # noqa: E731
    for f in (quant, back):
        assert f(x=None) == f(c=None) == f(s=None) == f(M=-1) == f(K=0) == f(ld=32) == ss.INVALID_ARG
        assert f(K=48) == f(M=1 << 50) == ss.UNSUPPORTED
        assert f(x=FAKE + 2) == f(ld=68) == f(c=FAKE + 2) == ss.MISALIGNED
        assert f(M=0) == ss.OK


def test_gemm_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = ss.MX4(FAKE, FAKE, 128, 64, 1, FAKE)

    def gemm(w=W, x=FAKE, M=4, ldx=128, y=FAKE, ldy=64, r=None, ldr=0, ws=FAKE, size=BIG):
        return status(lib, "mx4_gemm", ctypes.byref(w) if w else None, x, M, ldx, y, ldy, r, ldr, ws, size)

    assert gemm(w=None) == gemm(x=None) == gemm(y=None) == gemm(ws=None) == ss.INVALID_ARG
    assert gemm(w=ss.MX4(FAKE, FAKE, 128, 64, 1, None)) == gemm(w=ss.MX4(FAKE, FAKE, 128, 64, 2, FAKE)) == ss.INVALID_ARG
    assert gemm(M=-1) == gemm(ldx=120) == gemm(ldy=60) == gemm(r=FAKE + 64, ldr=60) == ss.INVALID_ARG
    assert gemm(r=FAKE, ldr=128) == ss.INVALID_ARG  # over y with another row length
    assert gemm(M=1 << 30) == ss.UNSUPPORTED
    assert gemm(x=FAKE + 2) == gemm(ldx=132) == gemm(y=FAKE + 4) == gemm(ldy=66) == gemm(ws=FAKE + 8) == ss.MISALIGNED
    assert gemm(r=FAKE + 4, ldr=64) == gemm(r=FAKE + 64, ldr=66) == gemm(w=ss.MX4(FAKE, FAKE, 128, 64, 1, FAKE + 8)) == ss.MISALIGNED
    assert gemm(size=lib.swiftspec_mx4_gemm_workspace_bytes(4, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL
    assert gemm(M=0) == ss.OK


def groups(ss, T=4, k=2, E=8, o=FAKE, r=FAKE, p=FAKE):  # noqa: F811
    return ctypes.byref(ss._Groups(T, k, E, o, r, p))


def bad_groups(ss):  # noqa: F811
    g = lambda **kw: groups(ss, **kw)  # noqa: E731
    return [(ss.INVALID_ARG, x) for x in (None, g(T=-1), g(k=0), g(E=0), g(k=9), g(o=None), g(r=None), g(p=None))] + \
        [(ss.UNSUPPORTED, x) for x in (g(E=513), g(k=17, E=32), g(T=1 << 28))] + \
        [(ss.MISALIGNED, x) for x in (g(o=FAKE + 2), g(r=FAKE + 1), g(p=FAKE + 2))]


def test_route_refusals(ss):  # noqa: F811
    lib = ss.lib()

    def route(g=groups(ss), x=FAKE, ld=8, e=FAKE, w=FAKE, ws=FAKE, size=BIG):
        return status(lib, "moe_route", x, ld, 1, e, w, g, ws, size)

    def group(g=groups(ss), e=FAKE, ws=FAKE, size=BIG):
        return status(lib, "moe_group", e, g, ws, size)

    for want, g in bad_groups(ss):
        assert route(g=g) == group(g=g) == want
    assert route(x=None) == route(e=None) == route(w=None) == route(ws=None) == route(ld=7) == ss.INVALID_ARG
    assert group(e=None) == group(ws=None) == ss.INVALID_ARG
    assert route(x=FAKE + 1) == route(e=FAKE + 2) == route(w=FAKE + 2) == group(e=FAKE + 2) == group(ws=FAKE + 2) == ss.MISALIGNED
    small = lib.swiftspec_moe_route_workspace_bytes(4, 8, 2) - 1
    assert route(size=small) == group(size=small) == ss.WORKSPACE_TOO_SMALL


def test_experts_refusals(ss):  # noqa: F811
    lib = ss.lib()
    W = lambda K=128, N=64, E=8, packed=FAKE: ctypes.byref(ss.MX4(FAKE, FAKE, K, N, E, packed))  # noqa: E731

    def swiglu(w=W(), u=W(), x=FAKE, ldx=128, g=groups(ss), h=FAKE, ldh=64, ws=FAKE, size=BIG):
        return status(lib, "moe_mx4_swiglu", w, u, x, ldx, g, h, ldh, ws, size)

    def down(w=W(), h=FAKE, ldh=128, g=groups(ss), p=FAKE, y=FAKE, ldy=64, r=None, ldr=0, ws=FAKE, size=BIG):
        return status(lib, "moe_mx4_down", w, h, ldh, g, p, y, ldy, r, ldr, ws, size)

    for want, g in bad_groups(ss):
        assert swiglu(g=g) == down(g=g) == want
    for f in (swiglu, down):
        assert f(w=None) == f(h=None) == f(ws=None) == f(ldh=56) == f(w=W(packed=None)) == f(w=W(E=7)) == ss.INVALID_ARG
        assert f(h=FAKE + 2) == f(ldh=130) == f(ws=FAKE + 8) == ss.MISALIGNED
        assert f(g=groups(ss, T=0)) == ss.OK
    assert swiglu(x=None) == swiglu(u=None) == swiglu(u=W(K=256)) == swiglu(u=W(N=32)) == swiglu(ldx=120) == ss.INVALID_ARG
    assert swiglu(g=groups(ss, T=1 << 26, k=1)) == down(g=groups(ss, T=1 << 26, k=1)) == ss.UNSUPPORTED
    assert swiglu(x=FAKE + 2) == swiglu(ldx=132) == ss.MISALIGNED
    assert down(p=None) == down(y=None) == down(ldy=60) == down(r=FAKE, ldr=128) == down(r=FAKE + 64, ldr=60) == ss.INVALID_ARG
    assert down(y=FAKE + 4) == down(ldy=66) == down(p=FAKE + 2) == down(r=FAKE + 4, ldr=64) == down(r=FAKE + 64, ldr=66) == ss.MISALIGNED
    assert swiglu(size=lib.swiftspec_moe_mx4_swiglu_workspace_bytes(4, 2, 8, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL
    assert down(size=lib.swiftspec_moe_mx4_down_workspace_bytes(4, 2, 8, 128, 64) - 1) == ss.WORKSPACE_TOO_SMALL


def test_reference_quantization():
    # every code of a block whose scale is 1, and the ties between them
    x = np.zeros((1, 32), np.float16)
    x[0, :16] = [4, 6, 5, -5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, 0.26, 7, 7.99, 0.5, -6]
    codes, scales = ref.quantize(x)
    assert scales.tolist() == [[127]]
    assert ref.values(codes, scales)[0, :16].tolist() == [4, 6, 4, -4, 0, 1, 1, 2, 2, 4, 0, 0.5, 6, 6, 0.5, -6]
    # homogeneous under powers of two, and at most a quarter of the largest off
    rng = np.random.default_rng(0)
    v = rng.standard_normal((5, 96)).astype(np.float16)
    q = ref.quantized(v)
    assert np.array_equal(ref.quantized(v * np.float16(0.25)), q / 4)
    assert np.abs(q - v).max() <= np.abs(v.astype(np.float64)).max() / 4


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (9, 4, 2), (30, 7, 7)])
def test_reference_routing(T, E, k):
    rng = np.random.default_rng(T)
    x = rng.standard_normal((T, E)).astype(np.float16)
    x[T // 2] = -np.inf
    experts, weights = ref.route(x, k)
    _, plain = ref.route(x, k, renormalize=False)
    live = np.arange(T) != T // 2
    assert np.allclose(weights[live].sum(-1), 1) and (experts[T // 2] == -1).all() and (weights[T // 2] == 0).all()
    assert (plain[live].sum(-1) <= 1 + 1e-12).all() and (k < E or np.allclose(plain[live].sum(-1), 1))
    offsets, rows, pos = ref.group(experts, E)
    assert offsets[-1] == k * live.sum()
    for p in range(T * k):
        if pos[p] >= 0:
            e = experts.reshape(-1)[p]
            assert rows[pos[p]] == p and offsets[e] <= pos[p] < offsets[e + 1]
    for e in range(E):
        assert (np.diff(rows[offsets[e]:offsets[e + 1]]) > 0).all()


def test_reference_block_of_one_expert_is_a_dense_one():
    """One expert of weight 1 for every token: the block is the SwiGLU and a
    product, and the places are the tokens."""
    rng = np.random.default_rng(1)
    T, H, F = 6, 64, 32
    x = rng.standard_normal((T, H)).astype(np.float16)
    wg, wu, wd = (ref.values(*ref.random_matrix(rng, 1, *s)) for s in ((F, H), (F, H), (H, F)))
    offsets, rows, pos = ref.group(np.zeros((T, 1), np.int32), 1)
    h, _ = ref.swiglu(x, wg, wu, offsets, rows, 1)
    g, u = ref.quantized(x) @ wg[0].T, ref.quantized(x) @ wu[0].T
    assert np.allclose(h, g / (1 + np.exp(-g)) * u)
    h16 = h.astype(np.float16)
    y, _ = ref.down(h16, wd, offsets, pos, np.ones((T, 1), np.float32))
    assert np.allclose(y, ref.gemm(h16, wd[0])[0])


def test_launches_of_too_many_threads(ss):  # noqa: F811
    """Sizes whose launch would reach 2^32 threads are refused, whatever memory the
    caller names for them."""
    lib = ss.lib()
    W = lambda K, N, E: ss.MX4(FAKE, FAKE, K, N, E, FAKE)  # noqa: E731
    G = lambda T, k, E: ss._Groups(T, k, E, FAKE, FAKE, FAKE)  # noqa: E731
    r = ctypes.byref
    # 512 matrices of 65536 x 4096: 72 GB packed
    assert status(lib, "mx4_prepack", r(W(65536, 4096, 512)), FAKE, BIG) == ss.UNSUPPORTED
    rows = (1 << 35) // 64
    assert status(lib, "mx4_quantize", FAKE, rows, 64, 64, FAKE, FAKE) == ss.UNSUPPORTED
    assert status(lib, "mx4_dequantize", FAKE, FAKE, rows, 64, FAKE, 64) == ss.UNSUPPORTED
    # at most 504 rows of 512 experts over 2^19 columns: up to 535 blocks of 16 rows
    assert status(lib, "moe_mx4_swiglu", r(W(128, 1 << 19, 512)), r(W(128, 1 << 19, 512)), FAKE, 128, r(G(63, 8, 512)), FAKE, 1 << 19,
                  FAKE, BIG) == ss.UNSUPPORTED
    # four results a thread of the combination
    assert status(lib, "moe_mx4_down", r(W(128, 8192, 8)), FAKE, 128, r(G(1 << 20, 1, 8)), FAKE, FAKE, 8192, None, 0, FAKE,
                  BIG) == ss.UNSUPPORTED


def test_tensors_that_the_library_would_read_differently(ss):  # noqa: F811
    """The binding refuses another type of the same width, sizes and strides that a
    32-bit number does not hold, and a matrix on another GPU."""
    torch = pytest.importorskip("torch")

    def refused(status, f, *args, **named):
        with pytest.raises(ss.SwiftSpecError) as e:
            f(*args, **named)
        assert e.value.status == status

    bad, big = ss.INVALID_ARG, ss.UNSUPPORTED
    t = lambda shape, stride, dtype: torch.empty_strided(shape, stride, dtype=dtype, device="meta")  # noqa: E731
    half, wide = torch.float16, (1 << 32) + 64
    assert ss._rows(t((3, 64), (72, 1), half), "", 64) == (3, 72)
    assert ss._rows(t((1, 64), (wide, 1), half), "", 64, 2**63 - 1) == (1, wide)
    for dtype in (torch.bfloat16, torch.int16, torch.float32):
        refused(bad, ss._rows, t((3, 64), (64, 1), dtype), "", 64)
    refused(big, ss._rows, t((2, 64), (wide, 1), half), "", 64)
    refused(big, ss._rows, t((1 << 31, 64), (64, 1), half), "", 64)
    refused(bad, ss._dense, t((3, 2), (2, 1), torch.float32), "", (3, 2), 4, real=False)
    refused(bad, ss._dense, t((3, 2), (2, 1), torch.int32), "", (3, 2), 4, real=True)
    codes, scales = torch.zeros(16, 64, dtype=torch.uint8), torch.zeros(16, 4, dtype=torch.uint8)
    refused(bad, ss.make_mx4, codes, scales)  # not on a GPU

    class OnGpu:
        def get_device(self):
            return 1

    W = ss.MX4(FAKE, FAKE, 128, 16, 1, FAKE)
    assert ss._same_device("", W, OnGpu()) == 1  # made without tensors: not known
    W.device = 0
    refused(bad, ss._same_device, "", W, OnGpu())
    W.device = 1
    assert ss._same_device("", W, OnGpu(), None, OnGpu()) == 1
