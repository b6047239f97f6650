"""The experts of a mixture in 8 bits on the GPU against 64 bits, and the block as it is
used: router with scores, SwiGLU and down projection beside a shared expert."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_fp8 import matrix
from test_gpu_moe import CASES, experts_of, groups_of, same_groups
from test_gpu_moe_forms import expert_edges, sample
from test_gpu_mx4 import check, half, strided

pytestmark = pytest.mark.gpu

# widths that end inside a block of 128, rows that end inside one
CASES = CASES + [(1, 4, 2, 16, 16, "random"), (9, 5, 3, 144, 272, "padded"), (150, 6, 2, 1040, 400, "random"), (900, 3, 2, 400, 1168, "padded"),
                 (4500, 4, 2, 176, 2064, "padded")]


@pytest.mark.parametrize("T,E,k,K,N,kind", CASES)
def test_swiglu(T, E, k, K, N, kind):
    rng = np.random.default_rng(T + E + K)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    out = torch.full((T * k + 2, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_fp8_swiglu_workspace_bytes(T, k, E, K, N))
    ss.moe_fp8_swiglu(Wg, Wu, strided(x, 8), g, out[:T * k, :N], ws)
    n = offsets[-1]
    if n:
        places = sample(n, expert_edges(offsets), 800)
        check(out[torch.from_numpy(places).to(dev()), :N], *ref.swiglu(x, wg, wu, offsets, rows, k, places))
    assert (out[n:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    assert ss.read_device_error(ws) == 0


@pytest.mark.parametrize("T,E,k,K,N,kind", CASES)
@pytest.mark.parametrize("residual", [False, True])
def test_down(T, E, k, K, N, kind, residual):
    rng = np.random.default_rng(T + E + K + 1)
    W, keep, w = matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    h = rng.standard_normal((T * k, K)).astype(np.float16)
    h[offsets[-1]:] = np.nan  # rows behind the last do not enter
    p = rng.random((T, k)).astype(np.float32)
    r = rng.standard_normal((T, N)).astype(np.float16) if residual else None
    out = torch.full((T + 1, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_fp8_down_workspace_bytes(T, k, E, K, N))
    ss.moe_fp8_down(W, strided(h, 8), g, up(p), out[:T, :N], ws, residual=strided(r, 4) if residual else None)
    edges = np.asarray(expert_edges(offsets))
    tokens = sample(T, rows[edges] // k if edges.size else (), 500)
    check(out[torch.from_numpy(tokens).to(dev()), :N], *ref.down(h, w, offsets, pos, p, r, tokens))
    assert (out[T:] == 7).all() and (out[:, N:] == 7).all() and torch.isfinite(out).all()
    if residual:
        y = half(r)
        ss.moe_fp8_down(W, half(h), g, up(p), y, ws, residual=y)
        assert torch.equal(y, out[:T, :N])
    assert ss.read_device_error(ws) == 0


# rows quantised by the product, then by a launch before it
@pytest.mark.parametrize("T,E,k,K,N", [(1, 8, 2, 256, 48), (3, 4, 2, 512, 128), (4, 6, 2, 2048, 1024), (16, 3, 1, 128, 128), (40, 8, 2, 256, 96),
                                       (500, 3, 2, 256, 512)])
def test_swiglu_over_its_own_input(T, E, k, K, N):
    """h in the buffer of x, from its start and from the middle of it."""
    rng = np.random.default_rng(K + T)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, "random"), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    ws = ss.workspace(ss.moe_fp8_swiglu_workspace_bytes(T, k, E, K, N))
    want = ref.swiglu(x, wg, wu, offsets, rows, k)
    for at in (0, 8 * (T * K // 16)):  # where h begins
        room = torch.zeros(max(T * K, at + T * k * N), dtype=torch.float16, device=dev())
        mine, out = room[:T * K].view(T, K), room[at:at + T * k * N].view(T * k, N)
        mine.copy_(half(x))
        ss.moe_fp8_swiglu(Wg, Wu, mine, g, out, ws)
        check(out, *want)
    assert ss.read_device_error(ws) == 0


@pytest.mark.parametrize("T", [6, 200])
def test_groups_that_do_not_hold(T):
    """Offsets, rows and places out of range set the error word, and nothing is
    written for them."""
    rng = np.random.default_rng(2)
    E, k, K, N = 3, 2, 128, 32
    (Wg, k1, wg), (Wu, k2, wu), (Wd, k3, wd) = (matrix(rng, E, *s) for s in ((N, K), (N, K), (N, K)))
    offsets, rows, pos = ref.group(experts_of(rng, T, E, k, "random"), E)
    x = half(rng.standard_normal((T, K)))
    hin = rng.standard_normal((T * k, K)).astype(np.float16)
    p = rng.random((T, k)).astype(np.float32)
    ws = ss.workspace(max(ss.moe_fp8_swiglu_workspace_bytes(T, k, E, K, N), ss.moe_fp8_down_workspace_bytes(T, k, E, K, N)))
    for i, v in ((0, 1), (1, -5), (2, T * k + 1), (3, T * k + 1), (1, 2 ** 31 - 1), (3, -1)):
        o = offsets.copy()
        o[i] = v
        g = ss.MoeGroups(T, k, E, up(o), up(rows), up(pos))
        h = torch.full((T * k, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_fp8_swiglu(Wg, Wu, x, g, h, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS and (h == 7).all()
        y = torch.full((T, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_fp8_down(Wd, half(hin), g, up(p), y, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS and (y == 7).all()
    want, bound = ref.swiglu(x.cpu().numpy(), wg, wu, offsets, rows, k)
    for v in (-1, T * k, 2 ** 31 - 1):
        r = rows.copy()
        r[3] = v
        g = ss.MoeGroups(T, k, E, up(offsets), up(r), up(pos))
        h = torch.full((T * k, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_fp8_swiglu(Wg, Wu, x, g, h, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS
        keep = np.arange(T * k) != 3
        check(h[torch.from_numpy(keep).to(dev())], want[keep], bound[keep])
        assert (h[3] == 7).all()
    for v in (T * k, 2 ** 31 - 1):
        q, without = pos.copy(), pos.copy()
        q[4], without[4] = v, -1
        g = ss.MoeGroups(T, k, E, up(offsets), up(rows), up(q))
        y = torch.empty(T, N, dtype=torch.float16, device=dev())
        ss.moe_fp8_down(Wd, half(hin), g, up(p), y, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS
        check(y, *ref.down(hin, wd, offsets, without, p))


class Block:
    """A mixture's feed-forward block as a program keeps it: an fp16 router, a shared
    expert that every token passes (a mixture of one), the experts, buffers and one
    workspace for a number of tokens."""

    def __init__(self, rng, T, E, k, H, F, **how):
        self.T, self.E, self.k, self.how = T, E, k, how
        self.Wr = half(rng.standard_normal((E, H)) / 16)
        self.bias = rng.standard_normal(E).astype(np.float32) * np.float32(0.1)
        self.scoring = ss.MoeScoring("sigmoid", bias=up(self.bias), **how)
        (self.Wg, k1, self.wg), (self.Wu, k2, self.wu), (self.Wd, k3, self.wd) = matrix(rng, E, F, H), matrix(rng, E, F, H), matrix(rng, E, H, F)
        (self.Sg, k4, self.sg), (self.Su, k5, self.su), (self.Sd, k6, self.sd) = matrix(rng, 1, F, H), matrix(rng, 1, F, H), matrix(rng, 1, H, F)
        self.keep = k1, k2, k3, k4, k5, k6
        self.gamma = half(rng.normal(1, 0.02, H))
        new = lambda *s, t=torch.float16: torch.zeros(*s, dtype=t, device=dev())  # noqa: E731
        self.xn, self.logits, self.h, self.hs = new(T, H), new(T, E, t=torch.float32), new(T * k, F), new(T, F)
        self.experts, self.weights = new(T, k, t=torch.int32), new(T, k, t=torch.float32)
        self.g = ss.MoeGroups(T, k, E)
        self.one = ss.MoeGroups(T, 1, 1)
        sizes = [ss.moe_route_workspace_bytes(T, E, k), ss.moe_route_workspace_bytes(T, 1, 1)]
        for j, n in ((k, E), (1, 1)):
            sizes += [ss.moe_fp8_swiglu_workspace_bytes(T, j, n, H, F), ss.moe_fp8_down_workspace_bytes(T, j, n, F, H)]
        sizes.append(ss.fp8_gemm_workspace_bytes(T, F, H))
        self.ws = ss.workspace(max(sizes))
        ss.moe_group(new(T, 1, t=torch.int32), self.one, self.ws)  # every token to the one expert

    def run(self, hidden):
        ss.rmsnorm(hidden, self.gamma, self.xn)
        torch.matmul(self.xn.float(), self.Wr.float().T, out=self.logits)
        ss.moe_route_scored(self.logits, self.scoring, self.experts, self.weights, self.g, self.ws)
        ss.moe_fp8_swiglu(self.Sg, self.Su, self.xn, self.one, self.hs, self.ws)
        ss.moe_fp8_swiglu(self.Wg, self.Wu, self.xn, self.g, self.h, self.ws)
        ss.fp8_gemm(self.Sd, self.hs, hidden, self.ws, residual=hidden)
        ss.moe_fp8_down(self.Wd, self.h, self.g, self.weights, hidden, self.ws, residual=hidden)


@pytest.mark.parametrize("T,E,k,H,F,groups", [(1, 8, 2, 512, 224, 4), (37, 20, 3, 256, 96, 5), (64, 8, 2, 1024, 272, 2), (400, 12, 4, 256, 160, 3)])
def test_block(T, E, k, H, F, groups):
    """Each stage against 64 bits on the stage before it; the calls of this library
    replayed from a graph between eager runs."""
    rng = np.random.default_rng(T)
    how = dict(groups=groups, top_groups=2, group_best=2, renormalize=True, scale=2.5)
    b = Block(rng, T, E, k, H, F, **how)
    x = rng.standard_normal((T, H)).astype(np.float16)
    hidden = half(x)
    b.run(hidden)
    xn, logits, h, hs = (t.cpu().numpy() for t in (b.xn, b.logits, b.h, b.hs))
    want_e, want_w = ref.route(logits, k, "sigmoid", b.bias, **how)
    assert np.array_equal(b.experts.cpu().numpy(), want_e)
    offsets, rows, pos = ref.group(want_e, E)
    same_groups(b.g, (offsets, rows, pos))
    check(b.h[:offsets[-1]], *ref.swiglu(xn, b.wg, b.wu, offsets, rows, k))
    check(b.hs, *ref.swiglu(xn, b.sg, b.su, np.array([0, T]), np.arange(T), 1))
    mid = half(x)
    ss.fp8_gemm(b.Sd, b.hs, mid, b.ws, residual=mid)
    check(mid, *ref.gemm(hs, b.sd[0], x))
    check(hidden, *ref.down(h, b.wd, offsets, pos, b.weights.cpu().numpy(), mid.cpu().numpy()))

    def own(hidden):  # without the library product of the logits
        ss.moe_route_scored(b.logits, b.scoring, b.experts, b.weights, b.g, b.ws)
        ss.moe_fp8_swiglu(b.Sg, b.Su, hidden, b.one, b.hs, b.ws)
        ss.moe_fp8_swiglu(b.Wg, b.Wu, hidden, b.g, b.h, b.ws)
        ss.fp8_gemm(b.Sd, b.hs, hidden, b.ws, residual=hidden)
        ss.moe_fp8_down(b.Wd, b.h, b.g, b.weights, hidden, b.ws, residual=hidden)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        again = half(x)
        g = ss.Graph()
        g.begin()
        own(again)
        g.end()
        for i in range(3):  # other tokens, other groups: one graph serves them
            x2 = half(rng.standard_normal((T, H)))
            b.logits.copy_(up(rng.standard_normal((T, E)).astype(np.float32)))
            again.copy_(x2)
            g.launch()
            own(x2)
            st.synchronize()
            assert torch.equal(again, x2)
    assert ss.read_device_error(b.ws) == 0
