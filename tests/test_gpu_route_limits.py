"""The router with scores where its scale, bias and scores leave the usual range."""
import itertools

import numpy as np
import pytest
import torch

import fp8_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [np.inf, -np.inf, np.nan, 3e38, -2.0, 0.0])
@pytest.mark.parametrize("T", [7, 300])  # one launch, and two
def test_slots_without_an_expert_weigh_nothing(scale, T):
    """Weight 0 whatever the scale; the weights of chosen experts follow the formula."""
    rng = np.random.default_rng(T)
    E, k = 24, 5
    x = rng.standard_normal((T, E)).astype(np.float32)
    x[::3] = -np.inf           # padding
    x[1::3, 2:] = -np.inf      # two experts for five slots
    for score, renormalize, groups in itertools.product(("softmax", "sigmoid"), (True, False), (1, 4)):
        how = dict(score=score, renormalize=renormalize, groups=groups, top_groups=1 if groups == 1 else 2, scale=scale)
        g = ss.MoeGroups(T, k, E)
        experts, weights = torch.empty(T, k, dtype=torch.int32, device=dev()), torch.full((T, k), 99.0, device=dev())
        ss.moe_route_scored(up(x), ss.MoeScoring(**how), experts, weights, g, ss.workspace(ss.moe_route_workspace_bytes(T, E, k)))
        with np.errstate(invalid="ignore"):
            want_e, want_w = ref.route(x, k, **how)
        assert np.array_equal(experts.cpu().numpy(), want_e) and (want_e[::3] < 0).all() and (want_e[1::3, 2:] < 0).all()
        got = weights.cpu().numpy()
        assert (got[want_e < 0] == 0).all()
        there = want_e >= 0
        if np.isfinite(scale):
            assert (np.abs(got - want_w) <= ref.weight_bound(want_w)).all()
        else:  # every chosen score here is positive
            assert np.array_equal(got[there], np.full(there.sum(), scale, np.float32), equal_nan=True)


@pytest.mark.parametrize("lowest", [-3.4028234663852886e38, -2e38])
def test_groups_of_the_lowest_biases(lowest):
    """Experts put off by the type's lowest value: the sum of a group's two is -inf, which
    stands with the groups that have no expert, after every other."""
    E, k = 12, 4
    bias = np.zeros(E, np.float32)
    bias[3:6] = lowest
    x = np.zeros((5, E), np.float32)
    x[1, :3] = -np.inf          # group 0 has no expert
    x[2, 6:] = -np.inf          # only groups 0 and 1 have
    x[3, [0, 1, 2, *range(6, 12)]] = -np.inf
    x[4] = -np.inf
    for best, top in itertools.product((1, 2), (1, 2, 3)):
        how = dict(score="sigmoid", groups=4, top_groups=top, group_best=best)
        g = ss.MoeGroups(5, k, E)
        experts, weights = torch.empty(5, k, dtype=torch.int32, device=dev()), torch.empty(5, k, device=dev())
        ss.moe_route_scored(up(x), ss.MoeScoring(bias=up(bias), **how), experts, weights, g, ss.workspace(ss.moe_route_workspace_bytes(5, E, k)))
        with np.errstate(over="ignore"):
            want_e, want_w = ref.route(x, k, bias=bias, **how)
        assert np.array_equal(experts.cpu().numpy(), want_e)
        assert (np.abs(weights.cpu().numpy() - want_w) <= ref.weight_bound(want_w)).all()
        if top > 1:  # the put-off group only where nothing else is left
            assert not np.isin(want_e[0], (3, 4, 5)).any() and (want_e[2, :3] == (0, 1, 2)).all()
