"""Pins of the routing's definition (oracle/fp8.py) at its edges: values worked out by hand."""

import numpy as np

from oracle import fp8

INF = float("inf")


def test_shut_out_experts_leave_their_group_to_the_open_ones():
    z = [[5.0, 4.0, 0.0, 3.0]]
    experts, w, offsets, src, slot = fp8.route(z, 1, [-INF, -INF, 0, -INF], groups=2)
    assert experts.tolist() == [[2]] and w.tolist() == [[1.0]] and offsets.tolist() == [0, 0, 0, 1, 1]
    # groups {0, 1, 2}, {3, 4, 5} of sigmoids: one open expert of 0.9 against two of 0.3, then against two of 0.6
    s = np.array([[0.9, 0.5, 0.5, 0.3, 0.3, 0.5], [0.9, 0.5, 0.5, 0.6, 0.6, 0.5]])
    experts, *_ = fp8.route(np.log(s / (1 - s)), 1, [0, -INF, -INF, 0, 0, -INF], sigmoid=True, groups=2)
    assert experts.tolist() == [[0], [3]]


def test_a_wanted_expert_beside_a_shut_out_one():
    experts, *_ = fp8.route([[5.0, 4.0, 0.0, 3.0]], 1, [0, 0, INF, -INF], groups=2)
    assert experts.tolist() == [[2]]


def test_shut_out_experts_that_fill_up_have_no_weight():
    z = np.log([[1.0, 2, 3, 4]])
    for renormalise, first in ((True, 2.0), (False, 0.6)):
        experts, w, *_ = fp8.route(z, 3, [-INF, -INF, 0, -INF], renormalise=renormalise, scale=2.0)
        assert experts.tolist() == [[2, 0, 1]]
        np.testing.assert_allclose(w, [[first, 0, 0]], rtol=1e-15)
    experts, w, *_ = fp8.route(z, 2, [-INF] * 4, groups=2)
    assert experts.tolist() == [[0, 1]] and w.tolist() == [[0, 0]]
    # not even where the score is a NaN
    experts, w, *_ = fp8.route([[np.nan, 1.0]], 2, [-INF, 0], sigmoid=True)
    assert experts.tolist() == [[1, 0]] and w.tolist() == [[1, 0]]


def test_weights_of_scores_next_to_nothing():
    want = 1 / (1 + np.exp(-0.5))
    for below in (650, 700, 709, 712):
        experts, w, *_ = fp8.route([[0.0, -below, -below - 0.5]], 2, [-INF, 0, 0], scale=2.5)
        assert experts.tolist() == [[1, 2]]
        np.testing.assert_allclose(w, [[2.5 * want, 2.5 * (1 - want)]], rtol=1e-12)
