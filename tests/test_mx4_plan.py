"""CPU checks of the plans of the 4-bit products: the kernel instance that each
shape of the GPU tests runs, both sides of the plan's lines, and workspaces."""
import ctypes
import itertools
import random

import pytest

import test_gpu_moe
import test_gpu_moe_forms as forms
import test_gpu_mx4
from test_abi import ss  # noqa: F401  (fixture: the built library)

FORMS = ("raw", "stream", "stream 32", "tile 64", "tile 128", "tile 256")


class Plan(ctypes.Structure):
    """ss::Mx4Plan (mx4_internal.h)."""
    _fields_ = [("form", ctypes.c_int), ("tm", ctypes.c_int), ("split", ctypes.c_int)]


@pytest.fixture(scope="module")
def plan(ss):  # noqa: F811
    """plan(M, E, K, N, swiglu, grouped, raw=True): form and shares of K by the
    library's own plan (an internal C++ function of the shared library)."""
    f = ctypes.CDLL(ss.LIB_PATH)["_ZN2ss13plan_mx4_gemmEiiiibbb"]
    f.restype = Plan
    f.argtypes = [ctypes.c_int] * 4 + [ctypes.c_bool] * 3

    def of(M, E, K, N, swiglu, grouped, raw=True):
        p = f(M, E, K, N, swiglu, grouped, raw)
        assert p.tm == (16, 16, 32, 64, 128, 256)[p.form]
        return FORMS[p.form], p.split

    return of


@pytest.fixture(scope="module")
def sizes(ss):  # noqa: F811
    """Bytes of a product's fp32 results, exactly and the most of up to M rows."""
    lib = ctypes.CDLL(ss.LIB_PATH)
    out = {}
    for name, symbol, args in (("part", "_ZN2ss14mx4_part_bytesEiii", "iii"), ("part most", "_ZN2ss19mx4_part_bytes_mostEiii", "iii"),
                               ("rows", "_ZN2ss14mx4_rows_bytesEiiii", "iiii"), ("rows most", "_ZN2ss19mx4_rows_bytes_mostElii", "lii")):
        f = lib[symbol]
        f.restype = ctypes.c_size_t
        f.argtypes = [{"i": ctypes.c_int, "l": ctypes.c_int64}[a] for a in args]
        out[name] = f
    return out


def drawn(n, seed):
    """M, E, K, N over the range of the plan's lines (over their logarithms)."""
    rng = random.Random(seed)
    log = lambda lo, hi: round(2 ** rng.uniform(lo, hi))  # noqa: E731
    for _ in range(n):
        yield log(0, 16), log(0, 9), 32 * log(0, 10), 16 * log(0, 11)


def test_forms_of_one_matrix_and_of_experts(plan):
    """Every form that a product has a kernel for, and no other: 32 rows a
    workgroup are for one matrix with K whole, shares of K for the tiles."""
    seen = set()
    for M, E, K, N in drawn(60000, 1):
        for kind, swiglu, grouped in (("gemm", False, False), ("swiglu", True, True), ("down", False, True)):
            for raw in (False, True):
                form, split = plan(M, E if grouped else 1, K, N, swiglu, grouped, raw)
                assert 1 <= split <= max(1, (K + 511) // 512 // 2)
                assert split == 1 or (form.startswith("tile") and not swiglu), (M, E, K, N)
                assert form != "stream 32" or not grouped, (M, E, K, N)
                assert form != "raw" or raw
                seen.add((kind, form, split > 1))
    assert seen == {(kind, form, split) for kind in ("gemm", "swiglu", "down") for form in FORMS for split in (False, True)
                    if not (form == "stream 32" and kind != "gemm") and not (split and (form[:4] != "tile" or kind == "swiglu"))
                    and (kind, form, split) not in (("down", "tile 128", True), ("down", "tile 256", True))}


# Both sides of the plan's lines.
@pytest.mark.parametrize("M,K,N,form,split", [
    (8, 8192, 8192, "raw", 1), (8, 8192, 28672, "stream", 1), (9, 8192, 8192, "stream", 1), (16, 4096, 4096, "raw", 1), (17, 4096, 4096, "stream", 1),
    (128, 4096, 4096, "stream 32", 1), (129, 4096, 4096, "tile 64", 2), (32, 8192, 8192, "stream 32", 1), (32, 11008, 4096, "stream", 1),
    (32, 4096, 4096, "stream", 1), (32, 28672, 8192, "tile 64", 4), (32, 8192, 28672, "tile 64", 1),
    (256, 8192, 8192, "tile 64", 1), (257, 8192, 8192, "tile 128", 1), (128, 14336, 4096, "tile 64", 4), (256, 14336, 4096, "tile 128", 4),
    (384, 8192, 28672, "tile 256", 1), (192, 8192, 28672, "tile 128", 1), (1024, 28672, 8192, "tile 256", 2)])
def test_lines_of_one_matrix(plan, M, K, N, form, split):
    assert plan(M, 1, K, N, False, False) == (form, split)


@pytest.mark.parametrize("M,E,K,N,swiglu,form,split", [
    (16, 16, 1024, 1024, False, "raw", 1), (16, 16, 1024, 1024, True, "tile 64", 1), (16, 8, 4096, 14336, True, "stream", 1),
    (32, 8, 4096, 14336, True, "tile 64", 1), (127, 128, 1024, 512, True, "stream", 1), (128, 128, 1024, 512, True, "tile 64", 1),
    (64 * 95, 64, 2048, 1024, True, "tile 64", 1), (64 * 128, 64, 2048, 1024, True, "tile 128", 1),
    (64 * 511, 64, 2048, 1024, True, "tile 128", 1), (64 * 512, 64, 2048, 1024, True, "tile 256", 1),
    (64 * 512, 64, 1024, 2048, False, "tile 256", 1), (8 * 192, 8, 14336, 4096, False, "tile 256", 1),
    (10 * 899, 10, 5536, 864, False, "tile 256", 1), (8 * 200, 8, 8192, 2048, False, "tile 128", 1),
    (8 * 200, 8, 8192, 1536, False, "tile 64", 1),
    (28, 6, 4544, 1120, False, "tile 64", 4), (400, 8, 14336, 1024, False, "tile 64", 3)])
def test_lines_of_experts(plan, M, E, K, N, swiglu, form, split):
    assert plan(M, E, K, N, swiglu, True) == (form, split)


def test_workspaces_hold_what_the_plans_write(sizes):
    """The fp32 results of a product and of any with fewer rows fit what the
    workspace query counts for them, however many experts share the rows."""
    rng = random.Random(2)
    for M, E, K, N in drawn(60000, 3):
        fewer = rng.randint(1, M)
        assert sizes["part"](M, K, N) <= sizes["part most"](M, K, N), (M, K, N)
        assert sizes["part"](fewer, K, N) <= sizes["part most"](M, K, N), (fewer, M, K, N)
        assert sizes["rows"](M, E, K, N) <= sizes["rows most"](M, K, N), (M, E, K, N)
        assert sizes["rows"](fewer, E, K, N) <= sizes["rows most"](M, K, N), (fewer, M, E, K, N)
    split = [sizes["rows"](M, E, K, N) > 4 * M * N for M, E, K, N in drawn(2000, 4)]
    assert any(split) and not all(split)


def test_gpu_tests_of_one_matrix_reach_every_form(plan):
    """The shapes of the GPU tests, with and without a residual, run every form
    of a plain product, whole and with K in shares."""
    got = [plan(M, 1, K, N, False, False) for M, K, N in test_gpu_mx4.SIZES]
    runs = [(form, len(list(same))) for form, same in itertools.groupby(got, key=lambda p: (p[0], p[1] > 1))]
    assert runs == [(("raw", False), 9), (("stream", False), 10), (("tile 64", False), 1), (("tile 64", True), 1), (("tile 64", False), 1),
                    (("tile 64", True), 1), (("tile 64", False), 1), (("tile 128", False), 1), (("tile 64", True), 5), (("tile 128", False), 1),
                    (("tile 128", True), 1), (("tile 256", False), 1), (("tile 128", True), 1), (("tile 256", True), 1), (("stream", False), 2),
                    (("stream 32", False), 3)]


def test_gpu_tests_of_experts_reach_every_form(plan):
    want = {"raw": ("random", "padded", "none"), "stream": ("random", "twice"), "tile 64": ("random", "padded", "twice", "one"),
            "tile 128": ("padded",), "tile 256": ("random", "padded")}
    for swiglu in (True, False):
        got = {}
        for T, E, k, K, N, kind in test_gpu_moe.CASES:
            got.setdefault(plan(T * k, E, K, N, swiglu, True)[0], set()).add(kind)
        assert got == {form: set(kinds) for form, kinds in want.items()}


def test_gpu_tests_run_the_forms_they_name(plan):
    for T, E, k, K, N, kind, form in forms.SWIGLU:
        assert plan(T * k, E, K, N, True, True) == (form, 1), (T, E, k, K, N)
    for T, E, k, K, N, kind, form, split in forms.DOWN:
        assert plan(T * k, E, K, N, False, True) == (form, split), (T, E, k, K, N)
    for M, form in forms.LARGE:
        assert plan(M, 1, forms.LARGE_K, forms.LARGE_N, False, False) == (form, 1)
    # several scale words in every tile form, and stores past the caches (h of more than 32 MiB) in two
    for cases in (forms.SWIGLU, forms.DOWN):
        assert {c[6] for c in cases if c[3] > 1024} >= {"tile 64", "tile 128", "tile 256", "raw", "stream"}
    assert {c[6] for c in forms.SWIGLU if c[0] * c[2] * c[4] * 2 > 32 << 20} == {"tile 128", "tile 256"}
    T, E, k, H, F = forms.PROMPT
    assert plan(T * k, E, H, F, True, True) == ("tile 256", 1) and plan(T * k, E, F, H, False, True) == ("tile 128", 1)
