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
