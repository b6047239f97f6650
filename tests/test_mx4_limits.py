"""CPU checks of the microscaled 4-bit and mixture entry points at the edges of
what they accept: each line is refused, or answered rightly, by both the C calls
and their binding."""
import pytest

from test_abi import ss  # noqa: F401  (fixture: the built library)
from test_mx4_abi import BIG, FAKE, groups, status


def refused(ss, want, f, *args, **named):  # noqa: F811
    with pytest.raises(ss.SwiftSpecError) as e:
        f(*args, **named)
    assert e.value.status == want


def test_router_workspace_alignment(ss):  # noqa: F811
    """The counts of the router's second launch are read eight bytes at a time."""
    lib = ss.lib()
    for off in (1, 2, 4, 6, 12):
        assert status(lib, "moe_route", FAKE, 8, 1, FAKE, FAKE, groups(ss), FAKE + off, BIG) == ss.MISALIGNED
        assert status(lib, "moe_group", FAKE, groups(ss), FAKE + off, BIG) == ss.MISALIGNED
    small = lib.swiftspec_moe_route_workspace_bytes(4, 8, 2) - 1
    for off in (0, 8):  # aligned enough: the next check answers
        assert status(lib, "moe_route", FAKE, 8, 1, FAKE, FAKE, groups(ss), FAKE + off, small) == ss.WORKSPACE_TOO_SMALL
        assert status(lib, "moe_group", FAKE, groups(ss), FAKE + off, small) == ss.WORKSPACE_TOO_SMALL


def test_size_queries_outside_what_the_calls_take(ss):  # noqa: F811
    """Sizes that no call takes, up to the largest 32-bit numbers, get no packed
    bytes and a workspace of the header alone; the largest that they do take get
    their size, whose parts pass 32 bits."""
    lib, top, head = ss.lib(), 2**31 - 1, ss.WS_HEADER_BYTES
    packed = lambda K, N, E: E * N * (-(-K // 128) * 64 + -(-K // 512) * 16)  # noqa: E731
    for K, N, E in ((65536, 65536, 1), (2**22 - 32, 1600, 8), (128, 32 * 2**20, 17), (top // 32 * 32, 16 * 2, 0), (4096, 14336, 512)):
        want = packed(K, N, E) if E else 0
        assert lib.swiftspec_mx4_packed_bytes(K, N, E) == want < 2**36
    for K, N, E in ((top, 16, 1), (top // 32 * 32, 16, 1), (128, top, 1), (128, top // 16 * 16, 512), (top, top, 1), (top, top, top),
                    (131072, 131072, 1), (128, 16, 513), (128, 16, top), (65536, 4096, 512), (0, 16, 1), (128, -16, 1)):
        assert lib.swiftspec_mx4_packed_bytes(K, N, E) == 0, (K, N, E)
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    rows = 2**25 - 1  # of 128 columns: just below 2 GiB
    assert lib.swiftspec_mx4_gemm_workspace_bytes(rows, 128, 16) == head + up(rows * 64) + up(rows * 16)
    for M, K, N in ((rows + 1, 128, 16), (top, 128, 16), (1, top, 16), (top, top, top), (16, top // 32 * 32, 16), (1, 128, top), (-1, 128, 16)):
        assert lib.swiftspec_mx4_gemm_workspace_bytes(M, K, N) == head, (M, K, N)
    # 256 units and more, of 65535 / k tokens; E rounded up to 4
    assert lib.swiftspec_moe_route_workspace_bytes(2**28 - 1, 5, 1) == head + up(-(-(2**28 - 1) // 65535) * 8 * 2)
    assert lib.swiftspec_moe_route_workspace_bytes(2**24 - 1, 512, 16) == head + up(-(-(2**24 - 1) // 4095) * 512 * 2)
    for T, E, k in ((2**28, 5, 1), (top, 5, 1), (top, 512, 16), (2**24, 512, 16), (4, 513, 1), (4, top, 2), (4, 64, 17), (4, 64, top)):
        assert lib.swiftspec_moe_route_workspace_bytes(T, E, k) == head, (T, E, k)
    swiglu, down = lib.swiftspec_moe_mx4_swiglu_workspace_bytes, lib.swiftspec_moe_mx4_down_workspace_bytes
    T = 2**24 - 1
    assert swiglu(T, 16, 512, 128, 16) == head + up(T * 64) + up(T * 16) + up((T + 512 + 1) * 16)
    assert down(T, 2, 512, 128, 16) == head + up(2 * T * 64) + up(2 * T * 16) + up((2 * T // 16 + 512 + 1) * 16) + up(2 * T * 64)
    for T, k, E, K, N in ((2**28, 1, 8, 128, 16), (top, 16, 512, 128, 16), (top, top, top, top, top), (1, 1, 1, top, 16), (4, 2, 513, 128, 16),
                          (4, 17, 64, 128, 16), (4, 2, 8, 128, top), (2**25, 1, 8, 128, 16), (4, 2, 512, 65536, 4096)):
        assert swiglu(T, k, E, K, N) == down(T, k, E, K, N) == head, (T, k, E, K, N)
    assert down(2**24, 2, 8, 128, 16) == head < swiglu(2**24, 2, 8, 128, 16)  # its rows are the pairs


def test_numbers_of_more_than_32_bits(ss):  # noqa: F811
    """The binding hands the library 32-bit numbers: longer ones would lose their
    upper bits, and a call would answer for other sizes."""
    torch = pytest.importorskip("torch")
    wide = 1 << 32
    new = lambda *shape, dtype=torch.uint8: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    # one row of 2^32 + 32 columns is no row of 32
    K = wide + 32
    x, codes, scales = new(1, K, dtype=torch.float16), new(1, K // 2), new(1, K // 32)
    refused(ss, ss.UNSUPPORTED, ss.mx4_quantize, x, codes, scales)
    refused(ss, ss.UNSUPPORTED, ss.mx4_dequantize, codes, scales, x)
    # nor matrices of 2^32 + 16 rows, of 2^32 + 64 columns, or 2^32 + 1 of them
    for shape in ((wide + 16, 64), (16, wide // 2 + 32), (wide + 1, 16, 64)):
        refused(ss, ss.UNSUPPORTED, ss.make_mx4, new(*shape), new(*shape[:-1], shape[-1] // 16))
    for T, k, E in ((wide + 4, 1, 8), (4, wide + 1, 8), (4, 1, wide + 8)):
        lists = new(E + 1, dtype=torch.int32), new(T * k, dtype=torch.int32), new(T * k, dtype=torch.int32)
        refused(ss, ss.UNSUPPORTED, ss.MoeGroups, T, k, E, *lists)
    head = ss.WS_HEADER_BYTES
    for n in (wide + 128, wide * wide + 128, -wide + 128):
        assert ss.mx4_packed_bytes(n, 16) == ss.mx4_packed_bytes(128, n) == ss.mx4_packed_bytes(128, 16, n) == 0
        for f, args in ((ss.mx4_gemm_workspace_bytes, (4, 128, 16)), (ss.moe_route_workspace_bytes, (4, 8, 2)),
                        (ss.moe_mx4_swiglu_workspace_bytes, (4, 2, 8, 128, 16)), (ss.moe_mx4_down_workspace_bytes, (4, 2, 8, 128, 16))):
            for i in range(len(args)):
                assert f(*args[:i], n, *args[i + 1:]) == head, (f.__name__, i, n)
            assert f(*args) > head


def test_packed_copies_that_do_not_hold_the_matrix(ss, monkeypatch):  # noqa: F811
    """Products read mx4_packed_bytes of the copy that make_mx4 is given: a smaller
    or a strided one is refused."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(ss, "_same_device", lambda *a: 0)
    for shape in ((16, 64), (3, 32, 96)):
        codes, scales = torch.zeros(shape, dtype=torch.uint8), torch.zeros(*shape[:-1], shape[-1] // 16, dtype=torch.uint8)
        n = ss.mx4_packed_bytes(2 * shape[-1], shape[-2], shape[0] if len(shape) == 3 else 1)
        for packed in (torch.zeros(n - 1, dtype=torch.uint8), torch.zeros(0, dtype=torch.uint8), torch.zeros(2 * n, dtype=torch.uint8)[::2],
                       torch.zeros(n // 4 - 1, dtype=torch.int32), torch.zeros(1, dtype=torch.uint8).expand(n)):
            refused(ss, ss.INVALID_ARG, ss.make_mx4, codes, scales, packed)
        for packed in (torch.zeros(n, dtype=torch.uint8), torch.zeros(n + 16, dtype=torch.uint8), torch.zeros(n // 4, dtype=torch.int32)):
            assert ss.make_mx4(codes, scales, packed).packed == packed.data_ptr()


def test_stream_of_another_device(ss, monkeypatch):  # noqa: F811
    """A call launches on the GPU of its tensors: a stream of another one is
    refused, one that does not name its GPU (a bare handle) is taken at its word."""

    class Stream:
        cuda_stream = 0x77

    def on(index):
        s = Stream()
        s.device_index = index
        return s

    calls = []
    monkeypatch.setattr(ss, "_cuda", (lambda dev: 0x55, lambda: 1))  # the current stream, the current device
    launch = lambda *a: calls.append(a) or 0  # noqa: E731
    refused(ss, ss.INVALID_ARG, ss._run, "", launch, on(0), 1, "x")
    assert calls == []
    for stream, handle in ((on(1), 0x77), (Stream(), 0x77), (None, 0x55)):
        ss._run("", launch, stream, 1, "x")
        assert calls.pop() == ("x", handle)
