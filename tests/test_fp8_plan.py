"""CPU checks of the plans of the 8-bit products: the kernel that each shape of the GPU
tests runs, both sides of the plan's lines, and workspaces."""
import ctypes
import random

import pytest

import test_gpu_fp8
import test_gpu_fp8_forms as forms
import test_gpu_fp8_moe
from test_abi import ss  # noqa: F401  (fixture: the built library)
from test_mx4_plan import Plan

FORMS = ("raw", "stream", "stream 32", "tile 64", "tile 128 deep", "tile 128", "tile 256")


@pytest.fixture(scope="module")
def plan(ss):  # noqa: F811
    """plan(M, E, K, N, swiglu, grouped, raw=True): form and shares of K by the
    library's own plan (an internal C++ function of the shared library)."""
    f = ctypes.CDLL(ss.LIB_PATH)["_ZN2ss13plan_fp8_gemmEiiiibbb"]
    f.restype = Plan
    f.argtypes = [ctypes.c_int] * 4 + [ctypes.c_bool] * 3

    def of(M, E, K, N, swiglu, grouped, raw=True):
        p = f(M, E, K, N, swiglu, grouped, raw)
        assert p.tm == (16, 16, 32, 64, 128, 128, 256)[p.form]
        return FORMS[p.form], p.split

    return of


@pytest.fixture(scope="module")
def sizes(ss):  # noqa: F811
    """Bytes of a product's fp32 results, exactly and the most of up to M rows."""
    lib = ctypes.CDLL(ss.LIB_PATH)
    out = {}
    for name, symbol, args in (("part", "_ZN2ss14fp8_part_bytesEiii", "iii"), ("part most", "_ZN2ss19fp8_part_bytes_mostEiii", "iii"),
                               ("rows", "_ZN2ss14fp8_rows_bytesEiiii", "iiii"), ("rows most", "_ZN2ss19fp8_rows_bytes_mostElii", "lii")):
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
        yield log(0, 16), log(0, 9), 16 * log(0, 11), 16 * log(0, 11)


def test_forms_of_one_matrix_and_of_experts(plan):
    """Every form that a product has a kernel for, and no other: 32 rows a workgroup are
    for one matrix with K whole, shares of K for tiles of up to 128 rows."""
    seen = set()
    for M, E, K, N in drawn(60000, 1):
        for kind, swiglu, grouped in (("gemm", False, False), ("swiglu", True, True), ("down", False, True)):
            for raw in (False, True):
                form, split = plan(M, E if grouped else 1, K, N, swiglu, grouped, raw)
                assert 1 <= split <= max(1, (K + 511) // 512 // 2)
                assert split == 1 or (form in ("tile 64", "tile 128 deep", "tile 128") and not swiglu), (M, E, K, N)
                assert form != "stream 32" or not grouped, (M, E, K, N)
                assert form != "raw" or (raw and M <= 16)
                seen.add((kind, form, split > 1))
    want = {(kind, form, False) for kind in ("gemm", "swiglu", "down") for form in FORMS if form != "stream 32" or kind == "gemm"}
    want |= {(kind, form, True) for kind in ("gemm", "down") for form in ("tile 64", "tile 128 deep")} | {("down", "tile 128", True)}
    assert want <= seen <= want | {("gemm", "tile 128", True)}


# Both sides of the plan's lines.
@pytest.mark.parametrize("M,K,N,form,split", [
    (8, 5120, 16384, "raw", 1), (9, 5120, 16384, "stream", 1), (16, 5136, 4096, "stream", 1), (8, 4096, 28672, "raw", 1), (8, 5120, 28672, "stream", 1),
    (8, 10240, 4096, "tile 64", 8), (8, 10224, 4096, "stream", 1), (8, 10240, 4112, "stream", 1), (9, 8192, 4096, "tile 64", 8),
    (9, 8176, 4096, "stream", 1), (16, 8192, 8192, "stream", 1), (17, 8192, 6144, "tile 64", 4), (16, 4096, 4096, "raw", 1), (16, 4096, 14336, "stream", 1),
    (17, 4096, 4096, "stream", 1), (32, 6144, 8192, "stream 32", 1), (32, 8192, 8192, "tile 64", 4), (16, 28672, 8192, "stream", 1),
    (32, 28672, 8192, "tile 64", 4), (32, 8192, 14336, "tile 64", 2), (64, 4096, 4096, "stream 32", 1), (65, 4096, 4096, "tile 64", 4),
    (64, 8192, 8192, "tile 64", 4), (256, 8192, 8192, "tile 64", 1), (512, 8192, 8192, "tile 128 deep", 1), (1024, 4096, 4096, "tile 128 deep", 1),
    (1500, 4096, 4096, "tile 128", 1), (1024, 8192, 8192, "tile 128", 1), (2048, 8192, 8192, "tile 256", 1), (4001, 4096, 14336, "tile 256", 1)])
def test_lines_of_one_matrix(plan, M, K, N, form, split):
    assert plan(M, 1, K, N, False, False) == (form, split)


@pytest.mark.parametrize("M,E,K,N,swiglu,form", [
    (16, 8, 4096, 14336, True, "raw"), (17, 8, 4096, 14336, True, "stream"), (31, 8, 4096, 14336, True, "stream"), (32, 8, 4096, 14336, True, "tile 64"),
    (9 * 64 - 1, 64, 2048, 1024, True, "stream"), (9 * 64, 64, 2048, 1024, True, "tile 64"), (64 * 128, 64, 2048, 1024, True, "tile 128"),
    (64 * 1024, 64, 2048, 1024, True, "tile 256"), (1400, 8, 4096, 14336, True, "tile 128"),
    (192, 8, 4096, 14336, True, "tile 64"), (256, 8, 4096, 14336, True, "tile 128"), (2048, 8, 4096, 14336, True, "tile 256"), (600, 5, 4096, 1024, True, "tile 64")])
def test_lines_of_experts(plan, M, E, K, N, swiglu, form):
    assert plan(M, E, K, N, swiglu, True) == (form, 1)


def test_workspaces_hold_what_the_plans_write(sizes):
    """The fp32 results of a product and of any with fewer rows fit what the workspace
    query counts for them, however many experts share the rows."""
    rng = random.Random(2)
    for M, E, K, N in drawn(60000, 3):
        fewer = rng.randint(1, M)
        assert sizes["part"](M, K, N) <= sizes["part most"](M, K, N), (M, K, N)
        assert sizes["part"](fewer, K, N) <= sizes["part most"](M, K, N), (fewer, M, K, N)
        assert sizes["rows"](M, E, K, N) <= sizes["rows most"](M, K, N), (M, E, K, N)
        assert sizes["rows"](fewer, E, K, N) <= sizes["rows most"](M, K, N), (fewer, M, E, K, N)
    split = [sizes["rows"](M, E, K, N) > 4 * M * N for M, E, K, N in drawn(2000, 4)]
    assert any(split) and not all(split)


def test_gpu_tests_run_the_forms_they_name(plan):
    for M, K, N, form, split in forms.GEMM:
        assert plan(M, 1, K, N, False, False) == (form, split), (M, K, N)
    for T, E, k, K, N, kind, form in forms.SWIGLU:
        assert plan(T * k, E, K, N, True, True) == (form, 1), (T, E, k, K, N)
    for T, E, k, K, N, kind, form, split in forms.DOWN:
        assert plan(T * k, E, K, N, False, True) == (form, split), (T, E, k, K, N)
    for M, form in forms.LARGE:
        assert plan(M, 1, forms.LARGE_K, forms.LARGE_N, False, False)[0] == form
    # in every form but two more than 64 groups of columns, whose scales a wave of a tile
    # loads anew, and few
    for cases, at in ((forms.GEMM, 3), (forms.SWIGLU, 6), (forms.DOWN, 6)):
        K = {"deep": {c[at] for c in cases if c[at - 2 - (at > 3)] > 8192}, "short": {c[at] for c in cases if c[at - 2 - (at > 3)] < 2048}}
        assert K["deep"] >= set(FORMS) - {"raw", "stream 32"}
        assert K["short"] >= {"raw", "tile 128 deep", "tile 128", "tile 256"}


def test_gpu_tests_reach_every_form(plan):
    got = {plan(M, 1, K, N, False, False)[0] for M, K, N in test_gpu_fp8.SIZES} | {c[3] for c in forms.GEMM}
    assert got == set(FORMS)
    for swiglu, named in ((True, forms.SWIGLU), (False, forms.DOWN)):
        got = {plan(T * k, E, K, N, swiglu, True)[0] for T, E, k, K, N, kind in test_gpu_fp8_moe.CASES} | {c[6] for c in named}
        assert got == set(FORMS) - {"stream 32"}
