"""The router with scores on the GPU against numpy: choices and groups exact, weights
to one rounding."""
import itertools

import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up
from test_gpu_moe import same_groups

pytestmark = pytest.mark.gpu


def rows_of(x, pad):
    """x on the GPU, in rows `pad` wider that hold larger scores behind."""
    t = torch.full((x.shape[0], x.shape[1] + pad), 99.0, dtype=torch.float16 if x.dtype == np.float16 else torch.float32, device=dev())
    t[:, :x.shape[1]] = up(x)
    return t[:, :x.shape[1]]


def check_route(x, k, pad=0, bias=None, **how):
    T, E = x.shape
    scoring = ss.MoeScoring(bias=None if bias is None else up(bias), **how)
    g = ss.MoeGroups(T, k, E)
    experts = torch.full((T, k), 99, dtype=torch.int32, device=dev())
    weights = torch.full((T, k), 99.0, device=dev())
    ss.moe_route_scored(rows_of(x, pad), scoring, experts, weights, g, ss.workspace(ss.moe_route_workspace_bytes(T, E, k)))
    want_e, want_w = ref.route(x, k, bias=bias, **how)
    assert np.array_equal(experts.cpu().numpy(), want_e)
    got = weights.cpu().numpy()
    assert (np.abs(got - want_w) <= ref.weight_bound(want_w)).all(), np.abs(got - want_w).max()
    same_groups(g, ref.group(want_e, E))
    return want_e, want_w


# T, E, k, groups, top_groups, padding of a row
SHAPES = [(1, 1, 1, 1, 1, 0), (1, 8, 2, 4, 2, 0), (1, 512, 16, 16, 4, 0), (7, 3, 3, 3, 2, 1), (63, 64, 8, 8, 3, 0), (64, 66, 6, 11, 5, 3),
          (65, 128, 1, 2, 1, 0), (129, 130, 5, 13, 13, 2), (300, 256, 8, 8, 4, 0), (1025, 2, 1, 2, 1, 0), (700, 60, 7, 1, 1, 4), (200, 512, 4, 512, 40, 0),
          (90, 96, 10, 32, 7, 5), (40, 48, 12, 6, 1, 0), (17, 160, 8, 8, 3, 0), (5000, 16, 4, 4, 2, 0), (33, 257, 3, 1, 1, 7)]


@pytest.mark.parametrize("T,E,k,groups,top_groups,pad", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_route(T, E, k, groups, top_groups, pad, score, dtype):
    rng = np.random.default_rng(T + E + k)
    # few distinct scores and biases: ties of experts and of groups; every fifth token, some scores and an expert masked
    x = (np.round(rng.standard_normal((T, E)) * 8) / 8).astype(dtype)
    x[rng.random((T, E)) < 0.2] = -np.inf
    x[4::5] = -np.inf
    bias = (np.round(rng.standard_normal(E) * 4) / 32).astype(np.float32)
    bias[E // 2] = -np.inf
    for n, (b, best, renormalize) in enumerate(itertools.product((None, bias), (1, 2), (True, False))):
        check_route(x, k, pad, b, score=score, groups=groups, top_groups=top_groups, group_best=best, renormalize=renormalize,
                    scale=(1.0, 2.5, -0.75)[n % 3])
    y = rng.standard_normal((T, E)).astype(dtype)
    check_route(y, k, pad, rng.standard_normal(E).astype(np.float32) * np.float32(0.1), score=score, groups=groups, top_groups=top_groups,
                group_best=2, renormalize=True, scale=1.0)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_at_their_limits(dtype, score):
    big = np.finfo(dtype).max
    x = np.zeros((9, 70), dtype)
    x[0] = -big            # the lowest finite value is a score like any other
    x[1, :] = -np.inf
    x[1, 69] = -big
    x[2, 5], x[2, 66] = np.inf, big   # +inf counts as the largest finite value: a tie
    x[3, 3] = np.nan
    x[4, ::2] = -0.0       # equal to 0
    x[5] = np.nan
    x[6, 1:] = dtype(2.0 ** -24)
    x[7] = np.arange(70) - 35
    x[8] = (np.arange(70) - 35) * 4  # gates of 0 and of 1
    bias = np.zeros(70, np.float32)
    bias[[3, 40, 41, 42, 43]] = np.inf, np.nan, -np.inf, -3.4e38, 3.4e38
    for b, n, renormalize in itertools.product((None, bias), (1, 5, 70), (True, False)):
        check_route(x, 6, 0, b, score=score, groups=n, top_groups=max(1, n // 3), group_best=2, renormalize=renormalize)


def test_close_scores_keep_their_order():
    """Scores a step apart in 32 bits, whose gates and sums with a bias are a step apart
    or equal."""
    rng = np.random.default_rng(8)
    x = np.float32(0.3) + np.arange(64, dtype=np.float32) * np.float32(2.0 ** -24)
    x = np.stack([rng.permutation(x) for _ in range(200)])
    for score in ("softmax", "sigmoid"):
        check_route(x, 8, score=score)
        check_route(x, 8, bias=np.full(64, 0.01, np.float32), score=score, groups=4, top_groups=2, group_best=2)


def test_softmax_without_groups_is_moe_route():
    rng = np.random.default_rng(2)
    T, E, k = 300, 72, 6
    x = rng.standard_normal((T, E)).astype(np.float16)
    experts, weights = check_route(x, k)
    g = ss.MoeGroups(T, k, E)
    e, w = torch.empty(T, k, dtype=torch.int32, device=dev()), torch.empty(T, k, device=dev())
    ss.moe_route(up(x), e, w, g, ss.workspace(ss.moe_route_workspace_bytes(T, E, k)))
    assert np.array_equal(e.cpu().numpy(), experts)
    assert np.abs(w.cpu().numpy() - weights).max() < 1e-6


def test_no_tokens_and_refusals():
    E, k = 12, 3
    ws = ss.workspace(ss.moe_route_workspace_bytes(4, E, k))
    new = lambda T: (torch.empty(T, k, dtype=torch.int32, device=dev()), torch.empty(T, k, device=dev()), ss.MoeGroups(T, k, E))  # noqa: E731
    e, w, g = new(0)
    ss.moe_route_scored(torch.empty(0, E, device=dev()), ss.MoeScoring(), e, w, g, ws)
    assert (g.offsets == 0).all()
    e, w, g = new(4)
    x = torch.zeros(4, E, device=dev())

    def refused(status, f):
        with pytest.raises(ss.SwiftSpecError) as err:
            f()
        assert err.value.status == status

    bad = ss.INVALID_ARG
    run = lambda x=x, s=ss.MoeScoring(), e=e, w=w, ws=ws: ss.moe_route_scored(x, s, e, w, g, ws)  # noqa: E731
    refused(bad, lambda: run(x=x.double()))
    refused(bad, lambda: run(x=x.to(torch.bfloat16)))
    refused(bad, lambda: run(x=x[:, :11]))
    refused(bad, lambda: run(x=x[:3]))
    refused(bad, lambda: run(x=x.T.contiguous().T))
    refused(bad, lambda: run(x=x.cpu()))
    refused(bad, lambda: run(e=e.long()))
    refused(bad, lambda: run(w=w.half()))
    refused(bad, lambda: run(s=ss.MoeScoring(groups=5)))                       # does not divide 12
    refused(bad, lambda: run(s=ss.MoeScoring(groups=4, top_groups=5)))
    refused(bad, lambda: run(s=ss.MoeScoring(group_best=3)))
    refused(bad, lambda: run(s=ss.MoeScoring(bias=torch.zeros(11, device=dev()))))
    refused(bad, lambda: ss.MoeScoring("tanh"))
    refused(bad, lambda: ss.MoeScoring(groups=0))
    refused(bad, lambda: ss.MoeScoring(bias=torch.zeros(12)))                  # not on the GPU
    refused(bad, lambda: ss.MoeScoring(bias=torch.zeros(24, device=dev())[::2]))
    refused(bad, lambda: ss.MoeScoring(bias=torch.zeros(12, dtype=torch.int32, device=dev())))
    refused(ss.WORKSPACE_TOO_SMALL, lambda: run(ws=ws[:1024]))
    run()
