"""The 8-bit products on the GPU in every form that their plan has, at columns and
depths that end inside a block and inside a scale word, against 64 bits for a sample
of rows and columns."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_moe import experts_of, groups_of
from test_gpu_moe_forms import expert_edges, sample
from test_gpu_mx4 import check, half, strided

pytestmark = pytest.mark.gpu


class Matrix:
    """E matrices of random codes (2^-4 and more, of either sign) and scales of any
    mantissa, and the values of a sample of their columns."""

    def __init__(self, seed, E, N, K, one=False, count=48):
        g = torch.Generator(device=dev())
        g.manual_seed(seed)
        shape = (N, K) if one else (E, N, K)
        codes = torch.randint(0x18, 0x58, shape, generator=g, device=dev(), dtype=torch.uint8)
        codes += 128 * torch.randint(0, 2, shape, generator=g, device=dev(), dtype=torch.uint8)
        scales = torch.exp2(torch.rand(*shape[:-2], -(-N // 128), -(-K // 128), generator=g, device=dev()) * 2 - 10)
        self.W = ss.make_fp8(codes, scales)
        self.keep = codes, scales, ss.prepack_fp8(self.W)
        # each block's first and last columns among them
        edges = np.concatenate([np.arange(0, N, 128), np.arange(127, N, 128)])
        at = np.random.default_rng(seed).choice(edges, min(count, edges.size), replace=False)
        self.at = np.unique(np.concatenate([at, sample(N, count=count, seed=seed)]))
        self.gpu_at = torch.from_numpy(self.at).to(dev())
        c = codes.index_select(-2, self.gpu_at).cpu().numpy()
        s = scales.cpu().numpy()
        self.values = ref.decoded(c) * np.repeat(s[..., self.at // 128, :].astype(np.float64), 128, -1)[..., :K]


# M, K, N, form, shares of K
GEMM = [(1, 5104, 144, "raw", 1), (1, 544, 144, "raw", 1), (1, 10384, 144, "tile 64", 8), (14, 9248, 4240, "stream", 1),
        (18, 9248, 144, "tile 64", 8), (17, 5408, 8752, "stream 32", 1), (37, 544, 4240, "stream 32", 1),
        (70, 528, 144, "tile 64", 1), (74, 8912, 144, "tile 64", 8), (131, 8640, 8384, "tile 64", 1), (137, 528, 11488, "tile 128 deep", 1),
        (137, 9360, 11168, "tile 128 deep", 1), (1193, 8656, 144, "tile 128 deep", 8), (1169, 528, 3392, "tile 128", 1), (2112, 8496, 2000, "tile 128", 1),
        (1292, 528, 6160, "tile 256", 1), (1309, 8496, 6160, "tile 256", 1)]


@pytest.mark.parametrize("M,K,N,form,split", GEMM)
@pytest.mark.parametrize("residual", [False, True])
def test_gemm_forms(M, K, N, form, split, residual):
    rng = np.random.default_rng(M + K)
    m = Matrix(M, 1, N, K, one=True)
    x = rng.standard_normal((M, K)).astype(np.float16)
    r = rng.standard_normal((M, N)).astype(np.float16) * 4 if residual else None
    out = torch.full((M + 1, N + 12), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N))
    ss.fp8_gemm(m.W, strided(x, 8), out[:M, :N], ws, residual=strided(r, 4) if residual else None)
    rows = sample(M)
    got = out[torch.from_numpy(rows).to(dev())][:, m.gpu_at]
    check(got, *ref.gemm(x[rows], m.values, r[np.ix_(rows, m.at)] if residual else None, ref.additions(K, split)))
    assert (out[M:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()


# T, E, k, K, N, kind, form
SWIGLU = [(1, 2, 2, 5104, 144, "random", "raw"), (1, 2, 2, 8464, 144, "random", "stream"),
          (7, 8, 2, 560, 144, "padded", "raw"), (9, 6, 2, 9232, 144, "padded", "stream"), (20, 2, 1, 9040, 144, "random", "tile 64"),
          (90, 4, 2, 528, 3536, "twice", "tile 128 deep"), (33, 2, 2, 10064, 5488, "random", "tile 128 deep"), (36, 2, 2, 576, 10896, "random", "tile 128"),
          (33, 2, 2, 9744, 11376, "padded", "tile 128"), (455, 12, 2, 544, 2640, "random", "tile 256"), (147, 3, 2, 9120, 8720, "random", "tile 256"),
          # h of more than 32 MiB, whose stores go past the caches
          (8000, 4, 2, 160, 1104, "padded", "tile 256"), (20000, 128, 2, 144, 1040, "padded", "tile 128")]


@pytest.mark.parametrize("T,E,k,K,N,kind,form", SWIGLU)
def test_swiglu_forms(T, E, k, K, N, kind, form):
    rng = np.random.default_rng(T + E + K)
    g, u = Matrix(T, E, N, K), Matrix(T + 1, E, N, K)
    u.at, u.gpu_at = g.at, g.gpu_at
    c = u.keep[0].index_select(-2, g.gpu_at).cpu().numpy()
    wu = ref.decoded(c) * np.repeat(u.keep[1].cpu().numpy()[..., g.at // 128, :].astype(np.float64), 128, -1)[..., :K]
    groups, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    out = torch.full((T * k + 2, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_fp8_swiglu_workspace_bytes(T, k, E, K, N))
    ss.moe_fp8_swiglu(g.W, u.W, strided(x, 8), groups, out[:T * k, :N], ws)
    n = offsets[-1]
    places = sample(n, expert_edges(offsets))
    got = out[torch.from_numpy(places).to(dev())][:, g.gpu_at]
    check(got, *ref.swiglu(x, g.values, wu, offsets, rows, k, places))
    assert (out[n:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    assert ss.read_device_error(ws) == 0


# T, E, k, K, N, kind, form, shares of K
DOWN = [(1, 2, 2, 5104, 160, "random", "raw", 1), (1, 2, 2, 8464, 160, "random", "stream", 1),
        (1, 16, 8, 1056, 528, "random", "raw", 1), (10, 9, 2, 8592, 144, "padded", "stream", 1),
        (56, 13, 1, 9888, 1184, "random", "tile 64", 1), (25, 1, 1, 9200, 144, "padded", "tile 64", 8), (43, 2, 2, 672, 11200, "padded", "tile 128 deep", 1),
        (35, 2, 2, 1712, 5616, "random", "tile 128 deep", 2), (502, 13, 2, 8496, 144, "padded", "tile 128 deep", 8),
        (1080, 47, 2, 544, 1136, "twice", "tile 128", 1), (749, 51, 4, 9440, 144, "random", "tile 128", 4), (601, 9, 2, 528, 4624, "padded", "tile 256", 1),
        (1558, 35, 2, 9248, 1680, "random", "tile 256", 1)]


@pytest.mark.parametrize("T,E,k,K,N,kind,form,split", DOWN)
@pytest.mark.parametrize("residual", [False, True])
def test_down_forms(T, E, k, K, N, kind, form, split, residual):
    rng = np.random.default_rng(T + E + K + 1)
    m = Matrix(T, E, N, K)
    groups, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    h = rng.standard_normal((T * k, K)).astype(np.float16)
    h[offsets[-1]:] = np.nan  # rows behind the last do not enter
    p = rng.random((T, k)).astype(np.float32)
    r = rng.standard_normal((T, N)).astype(np.float16) if residual else None
    out = torch.full((T + 1, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_fp8_down_workspace_bytes(T, k, E, K, N))
    ss.moe_fp8_down(m.W, strided(h, 8), groups, up(p), out[:T, :N], ws, residual=strided(r, 4) if residual else None)
    edges = np.asarray(expert_edges(offsets))
    tokens = sample(T, rows[edges] // k if edges.size else (), 100)
    got = out[torch.from_numpy(tokens).to(dev())][:, m.gpu_at]
    check(got, *ref.down(h, m.values, offsets, pos, p, r[:, m.at] if residual else None, tokens, ref.additions(K, split)))
    assert (out[T:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    assert ss.read_device_error(ws) == 0


# M rows of one matrix of more than 2 GiB, and the form
LARGE = [(5, "stream"), (40, "tile 64"), (100, "tile 128"), (300, "tile 128 deep"), (400, "tile 256")]
LARGE_K, LARGE_N = 49168, 49168


def test_matrix_of_more_than_2_gib():
    K, N = LARGE_K, LARGE_N
    m = Matrix(3, 1, N, K, one=True, count=40)
    assert m.keep[2].numel() > 2 ** 31
    rng = np.random.default_rng(12)
    for M, form in LARGE:
        print(M, form, flush=True)
        x = rng.standard_normal((M, K)).astype(np.float16)
        y = torch.full((M, N), float("nan"), dtype=torch.float16, device=dev())
        ss.fp8_gemm(m.W, half(x), y, ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N)))
        rows = sample(M, count=24)
        check(y[torch.from_numpy(rows).to(dev())][:, m.gpu_at], *ref.gemm(x[rows], m.values))
        assert torch.isfinite(y).all()


PROMPT = 1300, 4, 2, 1184, 1696


def test_block_of_prompts():
    """Router, SwiGLU and down at a prompt's size with padding, each stage within its
    bounds of 64 bits on the stage before it, replayed between eager runs on a
    workspace that two graphs share in turn."""
    rng = np.random.default_rng(21)
    T, E, k, H, F = PROMPT
    g, u, d = Matrix(1, E, F, H), Matrix(2, E, F, H), Matrix(3, E, H, F)
    full = [ref.values(w.keep[0].cpu().numpy(), w.keep[1].cpu().numpy()) for w in (g, u, d)]
    logits = up(rng.standard_normal((T, E)).astype(np.float32))
    logits[T - 50:] = float("-inf")  # padding
    scoring = ss.MoeScoring("sigmoid", bias=up(np.float32([0.1, 0, -0.1, 0])), groups=2, top_groups=2, group_best=1, scale=2.5)
    experts, weights = torch.empty(T, k, dtype=torch.int32, device=dev()), torch.empty(T, k, device=dev())
    groups = ss.MoeGroups(T, k, E)
    ws = ss.workspace(max(ss.moe_route_workspace_bytes(T, E, k), ss.moe_fp8_swiglu_workspace_bytes(T, k, E, H, F),
                          ss.moe_fp8_down_workspace_bytes(T, k, E, F, H)))
    h = torch.zeros(T * k, F, dtype=torch.float16, device=dev())

    def run(hidden):
        ss.moe_route_scored(logits, scoring, experts, weights, groups, ws)
        ss.moe_fp8_swiglu(g.W, u.W, hidden, groups, h, ws)
        ss.moe_fp8_down(d.W, h, groups, weights, hidden, ws, residual=hidden)

    x = rng.standard_normal((T, H)).astype(np.float16)
    hidden = half(x)
    run(hidden)
    offsets, rows, pos = ref.group(experts.cpu().numpy(), E)
    assert offsets[-1] == (T - 50) * k
    places, tokens = sample(offsets[-1], expert_edges(offsets)), sample(T)
    check(h[torch.from_numpy(places).to(dev())], *ref.swiglu(x, full[0], full[1], offsets, rows, k, places))
    check(hidden[torch.from_numpy(tokens).to(dev())],
          *ref.down(h.cpu().numpy(), full[2], offsets, pos, weights.cpu().numpy(), x, tokens))
    assert torch.equal(hidden[T - 50:], half(x[T - 50:]))  # padding keeps its residual
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        two, graphs = [half(x), half(x)], [ss.Graph(), ss.Graph()]
        for graph, again in zip(graphs, two):
            graph.begin()
            run(again)
            graph.end()
        for i in range(3):
            for graph, again in zip(graphs, two):
                x2 = half(rng.standard_normal((T, H)))
                again.copy_(x2)
                graph.launch()
                run(x2)
                st.synchronize()
                assert torch.equal(again, x2)
    assert ss.read_device_error(ws) == 0
