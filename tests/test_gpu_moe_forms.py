"""The experts of a mixture on the GPU at the sizes, layouts and kernel forms
that prompts and short calls use, against 64 bits."""
import numpy as np
import pytest
import torch

import mx4_bounds as bounds
import mx4_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_moe import experts_of, groups_of, same_groups
from test_gpu_mx4 import check, half, matrix, strided

pytestmark = pytest.mark.gpu


# rows quantised by the product, then by a launch before it
@pytest.mark.parametrize("T,E,k,K,N", [(1, 8, 2, 256, 48), (3, 4, 2, 512, 128), (4, 6, 2, 2048, 1024), (16, 3, 1, 128, 128), (40, 8, 2, 256, 96),
                                       (500, 3, 2, 256, 512)])
def test_swiglu_over_its_own_input(T, E, k, K, N):
    """h in the buffer of x, from its start and from the middle of it."""
    rng = np.random.default_rng(K + T)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, "random"), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    ws = ss.workspace(ss.moe_mx4_swiglu_workspace_bytes(T, k, E, K, N))
    want = ref.swiglu(x, wg, wu, offsets, rows, k)
    for at in (0, 8 * (T * K // 16)):  # where h begins
        room = torch.zeros(max(T * K, at + T * k * N), dtype=torch.float16, device=dev())
        mine, out = room[:T * K].view(T, K), room[at:at + T * k * N].view(T * k, N)
        mine.copy_(half(x))
        ss.moe_mx4_swiglu(Wg, Wu, mine, g, out, ws)
        check(out, *want)
    assert ss.read_device_error(ws) == 0


def sample(n, must=(), count=160, seed=0):
    """`count` of n rows, the first, the last and the given ones among them."""
    if n <= count:
        return np.arange(n)
    some = np.random.default_rng(seed).choice(n, count, replace=False)
    return np.unique(np.concatenate([some, [0, n - 1], np.asarray(must, int)]))


def expert_edges(offsets):
    """The first and the last place of each expert with any."""
    lo, hi = offsets[:-1], offsets[1:]
    return np.concatenate([lo[hi > lo], hi[hi > lo] - 1])


# K of several scale words (512 columns), with a last word and a last group that
# are not full, N no multiple of a tile: T, E, k, K, N, kind, form
SWIGLU = [(600, 8, 2, 2080, 1040, "padded", "tile 128"), (640, 5, 2, 1056, 1296, "random", "tile 128"), (1600, 3, 2, 2080, 1680, "padded", "tile 256"),
          (1600, 3, 2, 1056, 1744, "twice", "tile 256"), (90, 6, 3, 4640, 112, "padded", "tile 64"),
          # h of more than 32 MiB, whose stores go past the caches
          (4500, 4, 2, 160, 2064, "padded", "tile 256"), (20000, 128, 2, 96, 1040, "padded", "tile 128"),
          # few rows of long ones
          (1, 8, 2, 4128, 80, "random", "raw"), (9, 16, 2, 8224, 112, "padded", "stream")]


@pytest.mark.parametrize("T,E,k,K,N,kind,form", SWIGLU)
def test_swiglu_forms(T, E, k, K, N, kind, form):
    rng = np.random.default_rng(T + E + K)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    out = torch.full((T * k + 2, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_mx4_swiglu_workspace_bytes(T, k, E, K, N))
    ss.moe_mx4_swiglu(Wg, Wu, strided(x, 8), g, out[:T * k, :N], ws)
    n = offsets[-1]
    places = sample(n, expert_edges(offsets))
    check(out[torch.from_numpy(places).to(dev()), :N], *bounds.swiglu(x, wg, wu, offsets, rows, k, places, bounds.additions(K, form)))
    assert (out[n:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    assert ss.read_device_error(ws) == 0


# T, E, k, K, N, kind, form, shares of K
DOWN = [(600, 8, 2, 2080, 2064, "padded", "tile 128", 1), (640, 5, 2, 1056, 2576, "twice", "tile 128", 1), (1600, 3, 2, 2080, 3216, "padded", "tile 256", 1),
        (1600, 3, 2, 1056, 3472, "random", "tile 256", 1),
        # K in shares, several slots a token and tokens without any
        (70, 8, 3, 4640, 80, "padded", "tile 64", 5), (150, 4, 2, 3104, 336, "padded", "tile 64", 3), (90, 12, 9, 2208, 48, "twice", "tile 64", 2),
        # one token on its way back
        (1, 4, 2, 4128, 2064, "random", "raw", 1), (1, 16, 8, 1056, 528, "random", "raw", 1), (3, 8, 4, 4128, 1040, "padded", "stream", 1),
        (1, 5, 1, 96, 16, "none", "raw", 1)]


@pytest.mark.parametrize("T,E,k,K,N,kind,form,split", DOWN)
@pytest.mark.parametrize("residual", [False, True])
def test_down_forms(T, E, k, K, N, kind, form, split, residual):
    rng = np.random.default_rng(T + E + K + 1)
    W, keep, w = matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    h = rng.standard_normal((T * k, K)).astype(np.float16)
    h[offsets[-1]:] = np.nan  # rows behind the last do not enter
    p = rng.random((T, k)).astype(np.float32)
    r = rng.standard_normal((T, N)).astype(np.float16) if residual else None
    out = torch.full((T + 1, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_mx4_down_workspace_bytes(T, k, E, K, N))
    ss.moe_mx4_down(W, strided(h, 8), g, up(p), out[:T, :N], ws, residual=strided(r, 4) if residual else None)
    edges = np.asarray(expert_edges(offsets))
    tokens = sample(T, rows[edges] // k if edges.size else ())
    check(out[torch.from_numpy(tokens).to(dev()), :N], *bounds.down(h, w, offsets, pos, p, r, tokens, bounds.additions(K, form, split)))
    assert (out[T:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    assert ss.read_device_error(ws) == 0


# M rows of one matrix of more than 2 GiB, and the form: loads past its last group
# meet other codes of it
LARGE = [(5, "stream"), (33, "tile 64"), (130, "tile 128"), (300, "tile 256")]
LARGE_K, LARGE_N = 65568, 65552


def test_matrix_of_more_than_2_gib():
    K, N = LARGE_K, LARGE_N
    gen = torch.Generator(device=dev())
    gen.manual_seed(11)
    pick = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=gen, device=dev(), dtype=torch.uint8)  # noqa: E731
    codes, scales = pick(0, 256, N, K // 2), pick(117, 120, N, K // 32)
    W = ss.make_mx4(codes, scales)
    packed = ss.prepack_mx4(W)
    assert packed.numel() > 2 ** 31
    columns = np.unique(np.concatenate([np.arange(0, N, 701), [1, 32767, 32768, N - 17, N - 1]]))
    at = torch.from_numpy(columns).to(dev())
    w = ref.values(codes[at].cpu().numpy(), scales[at].cpu().numpy())
    rng = np.random.default_rng(12)
    for M, form in LARGE:
        print(M, form, flush=True)
        x = rng.standard_normal((M, K)).astype(np.float16)
        y = torch.full((M, N), float("nan"), dtype=torch.float16, device=dev())
        ss.mx4_gemm(W, half(x), y, ss.workspace(ss.mx4_gemm_workspace_bytes(M, K, N)))
        rows = sample(M, count=24)
        got, err = bounds.product(ref.quantized(x[rows]), w, bounds.additions(K, form))
        check(y[torch.from_numpy(rows).to(dev())][:, at], got, bounds.rounded(got, err))
        assert torch.isfinite(y).all()


# T, E, k, row length: aligned rows of more than 64 experts are read 16 bytes at a
# time, with whole and with partial last pieces; in one launch and in two
ALIGNED = [(1, 72, 8, 72), (90, 72, 3, 80), (700, 72, 8, 72), (33, 256, 8, 256), (3000, 256, 8, 264), (64, 260, 6, 264), (2000, 260, 4, 264),
           (5, 511, 16, 512), (4000, 512, 16, 512), (1500, 65, 2, 72), (200, 129, 5, 136), (500, 250, 7, 256)]


@pytest.mark.parametrize("T,E,k,ld", ALIGNED)
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_of_aligned_rows(T, E, k, ld, renormalize):
    rng = np.random.default_rng(T + E + k)
    # few distinct scores, whose differences are exact: ties; some masked, and whole tokens
    x = (np.round(rng.standard_normal((T, E)) * 8) / 8).astype(np.float16)
    x[rng.random((T, E)) < 0.2] = -np.inf
    x[4::5] = -np.inf
    x[:, E - 1] = np.where(rng.random(T) < 0.3, 4, x[:, E - 1])  # the last score counts
    want_e, want_w = ref.route(x, k, renormalize)
    logits = torch.full((T, ld), 9.0, dtype=torch.float16, device=dev())  # behind each row: larger scores
    logits[:, :E] = half(x)
    g = ss.MoeGroups(T, k, E)
    experts = torch.full((T, k), 99, dtype=torch.int32, device=dev())
    weights = torch.full((T, k), 99.0, device=dev())
    ss.moe_route(logits[:, :E], experts, weights, g, ss.workspace(ss.moe_route_workspace_bytes(T, E, k)), renormalize=renormalize)
    assert logits.data_ptr() % 16 == 0 and ld % 8 == 0
    assert np.array_equal(experts.cpu().numpy(), want_e)
    assert (np.abs(weights.cpu().numpy() - want_w) <= bounds.route_weights(want_w, E, renormalize)).all()
    same_groups(g, ref.group(want_e, E))


PROMPT = 1300, 4, 2, 1184, 1696


def test_block_of_prompts():
    """SwiGLU and down over one routing at a prompt's size, each stage within its
    bounds of 64 bits on the stage before it, replayed between eager runs."""
    rng = np.random.default_rng(21)
    T, E, k, H, F = PROMPT
    (Wg, k1, wg), (Wu, k2, wu), (Wd, k3, wd) = matrix(rng, E, F, H), matrix(rng, E, F, H), matrix(rng, E, H, F)
    logits = half(rng.standard_normal((T, E)))
    logits[T - 50:] = float("-inf")  # padding
    experts, weights = torch.empty(T, k, dtype=torch.int32, device=dev()), torch.empty(T, k, device=dev())
    g = ss.MoeGroups(T, k, E)
    ws = ss.workspace(max(ss.moe_route_workspace_bytes(T, E, k), ss.moe_mx4_swiglu_workspace_bytes(T, k, E, H, F),
                          ss.moe_mx4_down_workspace_bytes(T, k, E, F, H)))
    h = torch.zeros(T * k, F, dtype=torch.float16, device=dev())

    def run(hidden):
        ss.moe_route(logits, experts, weights, g, ws)
        ss.moe_mx4_swiglu(Wg, Wu, hidden, g, h, ws)
        ss.moe_mx4_down(Wd, h, g, weights, hidden, ws, residual=hidden)

    x = rng.standard_normal((T, H)).astype(np.float16)
    hidden = half(x)
    run(hidden)
    offsets, rows, pos = ref.group(experts.cpu().numpy(), E)
    same_groups(g, (offsets, rows, pos))
    places, tokens = sample(offsets[-1], expert_edges(offsets)), sample(T)
    check(h[torch.from_numpy(places).to(dev())], *bounds.swiglu(x, wg, wu, offsets, rows, k, places, bounds.additions(H, "tile 256")))
    check(hidden[torch.from_numpy(tokens).to(dev())],
          *bounds.down(h.cpu().numpy(), wd, offsets, pos, weights.cpu().numpy(), x, tokens, bounds.additions(F, "tile 128")))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        again = half(x)
        graph = ss.Graph()
        graph.begin()
        run(again)
        graph.end()
        for i in range(3):
            x2 = half(x) if i == 0 else half(rng.standard_normal((T, H)))
            again.copy_(x2)
            graph.launch()
            run(x2)
            st.synchronize()
            assert torch.equal(again, x2)
    assert ss.read_device_error(ws) == 0
