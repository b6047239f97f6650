"""The experts of a mixture on the GPU: routing and grouping against numpy, the
experts' products against 64 bits, and the block as it is used."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_mx4 import check, half, matrix, strided

pytestmark = pytest.mark.gpu


def route(logits, k, renormalize=True):
    T, E = logits.shape
    g = ss.MoeGroups(T, k, E)
    experts = torch.full((T, k), 99, dtype=torch.int32, device=dev())
    weights = torch.full((T, k), 99.0, device=dev())
    ws = ss.workspace(ss.moe_route_workspace_bytes(T, E, k))
    ss.moe_route(logits, experts, weights, g, ws, renormalize=renormalize)
    return experts, weights, g


def same_groups(g, want):
    for got, w, name in zip(g._tensors(), want, ("offsets", "rows", "pos")):
        assert np.array_equal(got.cpu().numpy(), w), name


ROUTES = [(1, 1, 1), (1, 8, 2), (1, 512, 16), (7, 3, 3), (63, 64, 8), (64, 65, 6), (65, 128, 1), (129, 130, 5),
          (1000, 256, 8), (1025, 2, 1), (3000, 60, 7), (20000, 512, 4),
          (70001, 13, 3), (96, 146, 10), (97, 146, 2), (256, 64, 4), (257, 64, 2), (1024, 4, 1), (640, 3, 2), (16385, 4, 4)]


@pytest.mark.parametrize("T,E,k", ROUTES)
@pytest.mark.parametrize("renormalize", [True, False])
def test_route(T, E, k, renormalize):
    rng = np.random.default_rng(T + E + k)
    # few distinct scores: ties; every fifth token and some experts masked
    x = (np.round(rng.standard_normal((T, E)) * 8) / 8).astype(np.float16)
    x[rng.random((T, E)) < 0.2] = -np.inf
    x[4::5] = -np.inf
    want_e, want_w = ref.route(x, k, renormalize)
    experts, weights, g = route(strided(x, 3), k, renormalize)
    assert np.array_equal(experts.cpu().numpy(), want_e)
    # exp, a sum of at most E / 64 + 6 + k levels and a division, each off by a few steps
    assert np.abs(weights.cpu().numpy() - want_w).max() <= (E / 64 + k + 16) * ref.STEP32
    same_groups(g, ref.group(want_e, E))


def test_route_scores_at_their_limits():
    x = np.zeros((8, 70), np.float16)
    x[0] = -65504           # the lowest finite value is a score like any other
    x[1, :] = -np.inf
    x[1, 69] = -65504
    x[2, 5], x[2, 66] = np.inf, 65504   # +inf counts as 65504: a tie
    x[3, 3] = np.nan
    x[4, ::2] = -0.0        # equal to 0
    x[5] = np.nan
    x[6, 1:] = np.float16(2.0 ** -24)
    x[7] = np.arange(70) - 35
    for renormalize in (True, False):
        want_e, want_w = ref.route(x, 4, renormalize)
        experts, weights, g = route(half(x), 4, renormalize)
        assert np.array_equal(experts.cpu().numpy(), want_e)
        assert np.abs(weights.cpu().numpy() - want_w).max() <= 24 * ref.STEP32
        same_groups(g, ref.group(want_e, 70))


@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (50, 7, 3), (300, 512, 16), (5000, 9, 2), (17000000, 5, 1)])
def test_group_of_given_experts(T, E, k):
    rng = np.random.default_rng(T)
    e = rng.integers(-2, E + 2, (T, k)).astype(np.int32)  # some without an expert
    e[:, -1] = e[:, 0]                                    # one named twice
    e[T // 2:] = E // 2                                   # a stretch of one expert
    g = ss.MoeGroups(T, k, E)
    ss.moe_group(up(e), g, ss.workspace(ss.moe_route_workspace_bytes(T, E, k)))
    same_groups(g, ref.group(e, E))


def test_no_tokens():
    g = ss.MoeGroups(0, 2, 5)
    ws = ss.workspace(1 << 17)
    ss.moe_group(torch.empty(0, 2, dtype=torch.int32, device=dev()), g, ws)
    assert (g.offsets == 0).all()
    ss.moe_route(torch.empty(0, 5, dtype=torch.float16, device=dev()), torch.empty(0, 2, dtype=torch.int32, device=dev()),
                 torch.empty(0, 2, device=dev()), g, ws)
    assert (g.offsets == 0).all()


def experts_of(rng, T, E, k, kind):
    if kind == "one":      # every token to one expert
        e = np.full((T, k), E - 1)
    elif kind == "twice":  # an expert named twice by a token
        e = rng.integers(0, E, (T, k))
        e[:, k - 1] = e[:, 0]
    else:
        p = np.exp(rng.standard_normal(E))
        e = np.stack([rng.choice(E, k, replace=False, p=p / p.sum()) for _ in range(T)])
        if kind == "padded":
            e[rng.random(T) < 0.3] = -1
    if kind == "none":
        e[:] = -1
    return e.astype(np.int32)


CASES = [(1, 1, 1, 32, 16, "random"), (1, 8, 2, 256, 48, "random"), (1, 64, 8, 2048, 64, "random"), (5, 4, 2, 160, 80, "padded"),
         (16, 8, 2, 1024, 32, "random"), (33, 5, 3, 96, 112, "twice"), (64, 2, 1, 512, 64, "one"), (64, 16, 4, 1408, 96, "padded"),
         (40, 300, 16, 128, 32, "random"), (7, 4, 2, 128, 32, "none"), (300, 3, 2, 352, 144, "random"), (600, 8, 2, 256, 272, "padded"),
         (700, 2, 2, 544, 80, "twice"), (513, 4, 1, 4096, 64, "one"),
         # fewer rows than experts, then enough tiles for the chip of 128 and of 256 rows
         (20, 64, 2, 256, 64, "random"), (30, 40, 4, 1056, 48, "twice"), (600, 8, 2, 96, 2064, "padded"),
         (1500, 3, 2, 160, 4112, "random"),
         # one slot a token: 64, 128 and 256 rows a tile
         (200, 5, 1, 256, 80, "padded"), (700, 6, 1, 96, 4112, "padded"), (2000, 3, 1, 64, 5136, "padded")]


def groups_of(e, E):
    T, k = e.shape
    want = ref.group(e, E)
    return ss.MoeGroups(T, k, E, *(up(a) for a in want)), want


@pytest.mark.parametrize("T,E,k,K,N,kind", CASES)
def test_swiglu(T, E, k, K, N, kind):
    rng = np.random.default_rng(T + E + K)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    e = experts_of(rng, T, E, k, kind)
    g, (offsets, rows, pos) = groups_of(e, E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    out = torch.full((T * k + 2, N + 4), 7.0, dtype=torch.float16, device=dev())
    h = out[:T * k, :N]
    ws = ss.workspace(ss.moe_mx4_swiglu_workspace_bytes(T, k, E, K, N))
    ss.moe_mx4_swiglu(Wg, Wu, strided(x, 8), g, h, ws)
    n = offsets[-1]
    if n:
        check(h[:n], *ref.swiglu(x, wg, wu, offsets, rows, k))
    assert (out[n:] == 7).all() and (out[:, N:] == 7).all()
    assert ss.read_device_error(ws) == 0


@pytest.mark.parametrize("T,E,k,K,N,kind", CASES)
@pytest.mark.parametrize("residual", [False, True])
def test_down(T, E, k, K, N, kind, residual):
    rng = np.random.default_rng(T + E + K + 1)
    W, keep, w = matrix(rng, E, N, K)
    e = experts_of(rng, T, E, k, kind)
    g, (offsets, rows, pos) = groups_of(e, E)
    h = rng.standard_normal((T * k, K)).astype(np.float16)
    h[offsets[-1]:] = np.nan  # rows behind the last do not enter
    p = rng.random((T, k)).astype(np.float32)
    r = rng.standard_normal((T, N)).astype(np.float16) if residual else None
    out = torch.full((T + 1, N + 4), 7.0, dtype=torch.float16, device=dev())
    ws = ss.workspace(ss.moe_mx4_down_workspace_bytes(T, k, E, K, N))
    ss.moe_mx4_down(W, strided(h, 8), g, up(p), out[:T, :N], ws, residual=strided(r, 4) if residual else None)
    check(out[:T, :N], *ref.down(h, w, offsets, pos, p, r))
    assert (out[T:] == 7).all() and (out[:, N:] == 7).all()
    if residual:
        y = half(r)
        ss.moe_mx4_down(W, half(h), g, up(p), y, ws, residual=y)
        assert torch.equal(y, out[:T, :N])
    assert ss.read_device_error(ws) == 0


@pytest.mark.parametrize("T", [6, 200])
def test_groups_that_do_not_hold(T):
    """Offsets, rows and places out of range set the error word, and nothing is
    written for them."""
    rng = np.random.default_rng(2)
    E, k, K, N = 3, 2, 128, 32
    (Wg, k1, wg), (Wu, k2, wu), (Wd, k3, wd) = (matrix(rng, E, *s) for s in ((N, K), (N, K), (N, K)))
    e = experts_of(rng, T, E, k, "random")
    offsets, rows, pos = ref.group(e, E)
    x = half(rng.standard_normal((T, K)))
    hin = rng.standard_normal((T * k, K)).astype(np.float16)
    p = rng.random((T, k)).astype(np.float32)
    ws = ss.workspace(max(ss.moe_mx4_swiglu_workspace_bytes(T, k, E, K, N), ss.moe_mx4_down_workspace_bytes(T, k, E, K, N)))
    for i, v in ((0, 1), (1, -5), (2, T * k + 1), (3, T * k + 1), (1, 2 ** 31 - 1), (3, -1)):
        o = offsets.copy()
        o[i] = v
        g = ss.MoeGroups(T, k, E, up(o), up(rows), up(pos))
        h = torch.full((T * k, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_mx4_swiglu(Wg, Wu, x, g, h, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS and (h == 7).all()
        y = torch.full((T, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_mx4_down(Wd, half(hin), g, up(p), y, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS and (y == 7).all()
    want, bound = ref.swiglu(x.cpu().numpy(), wg, wu, offsets, rows, k)
    for v in (-1, T * k, 2 ** 31 - 1):
        r = rows.copy()
        r[3] = v
        g = ss.MoeGroups(T, k, E, up(offsets), up(r), up(pos))
        h = torch.full((T * k, N), 7.0, dtype=torch.float16, device=dev())
        ss.moe_mx4_swiglu(Wg, Wu, x, g, h, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS
        keep = np.arange(T * k) != 3
        check(h[torch.from_numpy(keep).to(dev())], want[keep], bound[keep])
        assert (h[3] == 7).all()
    for v in (T * k, 2 ** 31 - 1):
        q, without = pos.copy(), pos.copy()
        q[4], without[4] = v, -1
        g = ss.MoeGroups(T, k, E, up(offsets), up(rows), up(q))
        y = torch.empty(T, N, dtype=torch.float16, device=dev())
        ss.moe_mx4_down(Wd, half(hin), g, up(p), y, ws)
        assert ss.read_device_error(ws) == ss.DEVERR_BAD_GROUPS
        check(y, *ref.down(hin, wd, offsets, without, p))


class Block:
    """A mixture's feed-forward block as a program keeps it: router and expert
    weights, buffers and one workspace for a number of tokens."""

    def __init__(self, rng, T, E, k, H, F):
        self.T, self.E, self.k = T, E, k
        (self.Wr, k0, self.wr) = matrix(rng, -(-E // 16) * 16, H)
        (self.Wg, k1, self.wg), (self.Wu, k2, self.wu), (self.Wd, k3, self.wd) = matrix(rng, E, F, H), matrix(rng, E, F, H), matrix(rng, E, H, F)
        self.keep = k0, k1, k2, k3
        self.gamma = rng.normal(1, 0.02, H).astype(np.float16)
        self.d_gamma = half(self.gamma)
        new = lambda *s, t=torch.float16: torch.zeros(*s, dtype=t, device=dev())  # noqa: E731
        self.xn, self.logits, self.h = new(T, H), new(T, self.Wr.N), new(T * k, F)
        self.experts, self.weights = new(T, k, t=torch.int32), new(T, k, t=torch.float32)
        self.g = ss.MoeGroups(T, k, E)
        self.ws = ss.workspace(max(ss.mx4_gemm_workspace_bytes(T, H, self.Wr.N), ss.moe_route_workspace_bytes(T, E, k),
                                   ss.moe_mx4_swiglu_workspace_bytes(T, k, E, H, F), ss.moe_mx4_down_workspace_bytes(T, k, E, F, H)))

    def run(self, hidden):
        ss.rmsnorm(hidden, self.d_gamma, self.xn)
        ss.mx4_gemm(self.Wr, self.xn, self.logits, self.ws)
        ss.moe_route(self.logits[:, :self.E], self.experts, self.weights, self.g, self.ws)
        ss.moe_mx4_swiglu(self.Wg, self.Wu, self.xn, self.g, self.h, self.ws)
        ss.moe_mx4_down(self.Wd, self.h, self.g, self.weights, hidden, self.ws, residual=hidden)


@pytest.mark.parametrize("T,E,k,H,F", [(1, 8, 2, 512, 224), (37, 20, 3, 256, 96), (64, 8, 2, 1024, 256), (400, 12, 4, 256, 160)])
def test_block(T, E, k, H, F):
    """Norm, router, routing and both halves of the experts, eager and replayed:
    each stage against 64 bits on the stage before it, every replay equal to the
    eager run."""
    rng = np.random.default_rng(T)
    b = Block(rng, T, E, k, H, F)
    x = rng.standard_normal((T, H)).astype(np.float16)
    hidden = half(x)
    b.run(hidden)
    xn, logits, h = (t.cpu().numpy() for t in (b.xn, b.logits, b.h))
    check(b.logits, *ref.gemm(xn, b.wr))
    want_e, want_w = ref.route(logits[:, :E], k)
    assert np.array_equal(b.experts.cpu().numpy(), want_e)
    offsets, rows, pos = ref.group(want_e, E)
    same_groups(b.g, (offsets, rows, pos))
    check(b.h, *ref.swiglu(xn, b.wg, b.wu, offsets, rows, k))
    check(hidden, *ref.down(h, b.wd, offsets, pos, b.weights.cpu().numpy(), x))

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        again = half(x)
        g = ss.Graph()
        g.begin()
        b.run(again)
        g.end()
        for i in range(3):  # other tokens, other groups: one graph serves them
            x2 = x if i == 0 else rng.standard_normal((T, H)).astype(np.float16)
            again.copy_(half(x2))
            g.launch()
            eager = half(x2)
            b.run(eager)
            st.synchronize()
            assert torch.equal(again, eager)
            if i == 0:
                assert torch.equal(again, hidden)
    assert ss.read_device_error(b.ws) == 0


def test_refusals_of_the_binding():
    rng = np.random.default_rng(4)
    E, T, k, K, N = 4, 3, 2, 64, 32
    (W, k1, _), (V, k2, _) = matrix(rng, E, N, K), matrix(rng, E + 1, N, K)
    g, _ = groups_of(experts_of(rng, T, E, k, "random"), E)
    ws = ss.workspace(1 << 20)
    x, h, y = (torch.zeros(n, m, dtype=torch.float16, device=dev()) for n, m in ((T, K), (T * k, N), (T, N)))
    hk = torch.zeros(T * k, K, dtype=torch.float16, device=dev())
    p = torch.zeros(T, k, device=dev())
    e = torch.zeros(T, k, dtype=torch.int32, device=dev())

    def refused(status, f):
        with pytest.raises(ss.SwiftSpecError) as err:
            f()
        assert err.value.status == status

    bad = ss.INVALID_ARG
    refused(bad, lambda: ss.moe_mx4_swiglu(W, V, x, g, h, ws))       # another number of experts
    refused(bad, lambda: ss.moe_mx4_swiglu(V, V, x, g, h, ws))
    refused(bad, lambda: ss.moe_mx4_swiglu(W, W, x[:2], g, h, ws))   # other tokens
    refused(bad, lambda: ss.moe_mx4_swiglu(W, W, x, g, h[:4], ws))
    refused(bad, lambda: ss.moe_mx4_down(W, hk, g, p[:2], y, ws))
    refused(bad, lambda: ss.moe_mx4_down(W, hk, g, p.double(), y, ws))
    refused(bad, lambda: ss.moe_mx4_down(W, hk, g, p, y[:2], ws))
    refused(ss.WORKSPACE_TOO_SMALL, lambda: ss.moe_mx4_down(W, hk, g, p, y, ws[:ss.moe_mx4_down_workspace_bytes(T, k, E, K, N) - 1]))
    refused(bad, lambda: ss.moe_route(torch.zeros(T, E + 1, dtype=torch.float16, device=dev()), e, p, g, ws))
    refused(bad, lambda: ss.moe_route(torch.zeros(T, E, device=dev()), e, p, g, ws))
    refused(bad, lambda: ss.moe_group(e.long(), g, ws))
    refused(bad, lambda: ss.MoeGroups(T, k, E, offsets=g.offsets[:-1]))
    refused(bad, lambda: ss.mx4_gemm(W, x, y, ws))                   # experts' weights in a plain product
    refused(bad, lambda: ss.moe_group(torch.zeros(T, 9, dtype=torch.int32, device=dev()), ss.MoeGroups(T, 9, E), ws))  # k > E
