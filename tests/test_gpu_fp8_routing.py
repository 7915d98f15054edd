"""Routing where scores are next to nothing, experts are shut out, or logits are infinite."""

import numpy as np
import pytest

from oracle import fp8
from tests.test_gpu_fp8_ops import check_route, metro, run_route  # noqa: F401

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -1074  # the spacing of fp64 below 2^-1022


def check_small(metro, z, k, bias, scoring, scale):
    """Scores below 2^-1022 are off by their spacing: by an exponential and a division of half a step each on either
    side, so a weight by twice that of its own score and of each of the sum's, beside its rounding to fp32."""
    got = run_route(metro, z, k, bias, scoring=scoring, scale=scale)
    z32 = z.astype(np.float32)
    want = fp8.route(z32, k, bias, bool(scoring), scale=scale)
    one = fp8.route(z32, k, bias, bool(scoring), renormalise=False)[1]
    np.testing.assert_array_equal(got[0], want[0])
    total = one.sum(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        off = np.where(total > 0, 2 * LEAST / one + 2 * k * LEAST / total, 0.0)
    assert np.isfinite(got[1]).all()
    assert np.all(np.abs(got[1] - want[1]) <= (2.0 ** -23 + off) * want[1])
    return got


@pytest.mark.parametrize("T", [1, 5, 9, 70, 2100])
@pytest.mark.parametrize("scale", [1.0, 2.5])
@pytest.mark.parametrize("below", [650, 700, 708.5, 709, 709.5, 712, 730, 740])
def test_route_scores_far_below_a_shut_out_maximum(metro, T, scale, below):
    z = np.zeros((T, 8))
    z[:] = [0, -below, -below - 0.5, -below - 1, -900, -900, -900, -900]
    z[1:] += np.arange(1, T)[:, None] % 4
    bias = np.zeros(8, np.float32)
    bias[0] = -np.inf
    got = check_small(metro, z, 2, bias, 0, scale)
    np.testing.assert_allclose(got[1].sum(1), scale, rtol=2.0 ** -22)


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("scale", [1.0, 2.5])
@pytest.mark.parametrize("below", [650, 700, 708.5, 709, 709.5, 712])
def test_route_sigmoids_next_to_nothing(metro, T, scale, below):
    """(Below -709.78 the exponential of the definition is infinite: scores and weights are 0.)"""
    z = np.tile([-below, -below - 0.125, -900, -900], (T, 1))
    got = check_small(metro, z, 2, None, 1, scale)
    np.testing.assert_allclose(got[1].sum(1), 0.0 if below > 709.8 else scale, rtol=2.0 ** -22)


# --- shut out experts ---------------------------------------------------------------


@pytest.mark.parametrize("T", [1, 8, 64, 65, 200, 2100])
@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("E,k,groups,top", [(4, 1, 2, 1), (8, 2, 2, 1), (8, 2, 4, 2), (8, 4, 1, 1), (16, 3, 16, 4), (32, 4, 8, 3), (64, 6, 32, 5),
                                            (128, 8, 8, 4), (256, 8, 64, 6), (512, 9, 8, 2)])
def test_route_shut_out_experts(metro, T, scoring, E, k, groups, top):
    """Of every group none to two are left open, of some runs of groups nothing."""
    rng = np.random.default_rng([T, E, groups, scoring])
    z, per = rng.normal(size=(T, E)) * 2, E // groups
    for open_ in (0, 1, 2):
        bias = np.full(E, -np.inf, np.float32)
        for g in range(groups):
            n = min(per, int(rng.integers(0, open_ + 1)))
            bias[g * per + rng.permutation(per)[:n]] = rng.normal(size=n) * 0.1
        got = check_route(metro, z, k, bias, scoring, groups, top, renormalise=open_ != 1, scale=1.5)
        shut = np.isneginf(bias)[got[0]]
        assert not got[1][shut].any()
        # where the experts left are enough, none that is shut out is chosen
        if groups == 1 or top == groups:
            assert shut.sum(1).tolist() == [max(0, k - int(np.isfinite(bias).sum()))] * T


@pytest.mark.parametrize("T", [3, 70])
def test_route_keeps_the_group_of_the_only_open_expert(metro, T):
    z = np.tile([5.0, 4, 0, 3], (T, 1))
    got = check_route(metro, z, 1, [-np.inf, -np.inf, 0, -np.inf], n_groups=2, top_groups=1)
    assert (got[0] == 2).all() and (got[1] == 1).all()
    got = check_route(metro, z, 2, [-np.inf, -np.inf, 0, -np.inf])
    assert (got[0] == [2, 0]).all() and (got[1] == [1, 0]).all()
    # a wanted expert beside a shut out one
    got = check_route(metro, z, 1, [0, 0, np.inf, -np.inf], n_groups=2, top_groups=1)
    assert (got[0] == 2).all()


@pytest.mark.parametrize("T", [3, 70])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_route_shut_out_experts_of_any_logit_have_no_weight(metro, T, value):
    z = np.tile([value, 1.0, value, 2.0], (T, 1))
    with np.errstate(all="ignore"):
        got = check_route(metro, z, 4, [-np.inf, 0, -np.inf, 0], scoring=1, scale=2.0)
        assert (got[0] == [3, 1, 0, 2]).all() and (got[1][:, 2:] == 0).all()
        check_route(metro, z, 4, [-np.inf, 0, -np.inf, 0], scoring=1, renormalise=False)


@pytest.mark.parametrize("T", [3, 70])
def test_route_infinite_logits(metro, T):
    """+inf in a softmax row makes its weights NaN, and under sigmoid a score of 1."""
    z = np.random.default_rng(T).normal(size=(T, 16))
    z[1, 4] = np.inf
    for groups, top in ((1, 1), (4, 2)):
        with np.errstate(all="ignore"):
            got = check_route(metro, z, 4, n_groups=groups, top_groups=top)
            assert np.isnan(got[1][1]).all() and np.isfinite(np.delete(got[1], 1, 0)).all()
            got = check_route(metro, z, 4, scoring=1, n_groups=groups, top_groups=top, renormalise=False)
            assert got[0][1, 0] == 4 and got[1][1, 0] == 1
