"""Pins of the routing's definition (oracle/fp8.py) at its edges: values worked out by hand."""

import numpy as np

from oracle import fp8

INF = float("inf")


def test_weights_of_scores_next_to_nothing():
    want = 1 / (1 + np.exp(-0.5))
    for below in (650, 700, 709, 712):
        experts, w, *_ = fp8.route([[0.0, -below, -below - 0.5]], 2, [-INF, 0, 0], scale=2.5)
        assert experts.tolist() == [[1, 2]]
        np.testing.assert_allclose(w, [[2.5 * want, 2.5 * (1 - want)]], rtol=1e-12)
