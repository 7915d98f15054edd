"""The oracle of the speculative decoding step's operators against closed forms and the model's own oracle."""

import math

import numpy as np
import pytest

from oracle import causal_gqa_attention, rms_norm
from oracle import draft as D


def test_rows_are_normalised_and_turned_by_pairs():
    rng = np.random.default_rng(1)
    nq, nkv, hd, base = 4, 2, 64, 1e4
    y = rng.standard_normal((5, (nq + 2 * nkv) * hd))
    pos = np.array([0, 1, 17, 99, 100])
    angle = np.arange(100)[:, None] * base ** (-2.0 * np.arange(hd // 2) / hd)
    rope = np.stack([np.cos(angle), np.sin(angle)], axis=2)
    g = 1 + 0.1 * rng.standard_normal(hd)
    q, k, v = D.rope_rows(y, nq, nkv, hd, g, None, 1e-5, rope, pos)
    heads = y.reshape(5, -1, hd)
    np.testing.assert_array_equal(v, heads[:, nq + nkv:])
    np.testing.assert_allclose(q[0], rms_norm(heads[0, :nq], g, 1e-5), rtol=1e-12)  # (position 0 turns nothing)
    np.testing.assert_allclose(np.hypot(k[2, 0, :32], k[2, 0, 32:]), np.hypot(heads[2, nq, :32], heads[2, nq, 32:]), rtol=1e-12)
    z = (heads[2, nq, :32] + 1j * heads[2, nq, 32:]) * np.exp(1j * angle[17])
    np.testing.assert_allclose(k[2, 0], np.concatenate([z.real, z.imag]), rtol=1e-10, atol=1e-12)
    assert np.isnan(q[4]).all() and np.isnan(k[4]).all() and np.isfinite(v[4]).all()


def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(2)
    q, K, V = rng.standard_normal((6, 8, 64)), rng.standard_normal((20, 4, 64)), rng.standard_normal((20, 4, 64))
    see = np.arange(20)[None] <= 14 + np.arange(6)[:, None]
    np.testing.assert_allclose(D.tree_attention(q, K, V, see), causal_gqa_attention(q, K, V, 14 + np.arange(6)), rtol=1e-12)


def test_unseen_keys_take_no_part():
    q, K, V = np.ones((2, 1, 64)), np.full((3, 1, 64), np.nan), np.full((3, 1, 64), np.inf)
    K[1], V[1] = 1.0, 5.0
    out = D.tree_attention(q, K, V, np.array([[False, True, False], [False] * 3]))
    assert (out[0] == 5.0).all() and (out[1] == 0.0).all()


@pytest.mark.parametrize("u,token", [(0.0, 2), (0.49, 2), (0.51, 0), (0.74, 0), (0.76, 3), (0.99, 3), (1.0, 3), (2.0, 3),
                                     (-1.0, 2), (math.nan, 2)])
def test_choice_by_running_sums(u, token):
    x = [math.log(2.0), -math.inf, math.log(4.0), math.log(2.0), math.nan]
    assert D.sample(x, u) == (token, pytest.approx(0.5 if token == 2 else 0.25))


def test_filters_keep_beginnings_of_the_order():
    x = np.log([1.0, 8.0, 4.0, 2.0, 1.0])
    last = lambda **kw: D.sample(x, 1.0, **kw)
    assert last() == (4, pytest.approx(1 / 16))
    assert last(top_k=2) == (2, pytest.approx(1 / 3))
    assert last(top_k=4) == (0, pytest.approx(1 / 15))  # (ties by the lowest index)
    assert last(top_p=0.5) == (1, 1.0)
    assert last(top_p=0.51) == (2, pytest.approx(1 / 3))
    assert last(top_p=0.0) == (1, 1.0)
    assert last(min_p=0.2) == (3, pytest.approx(1 / 7))
    assert last(min_p=0.2, top_k=2, top_p=0.7) == (2, pytest.approx(1 / 3))
    assert last(top_k=2, top_p=0.6) == (1, 1.0)  # (of the two that top-k leaves)
    assert last(temperature=0.5) == (4, pytest.approx(1 / 86))
    assert last(temperature=0.0) == (1, 1.0)
    assert last(temperature=math.nan) == (1, 1.0)
    assert last(temperature=math.inf) == (4, pytest.approx(0.2))
    assert D.sample([-math.inf, math.nan], 0.5) == (-1, 0.0)
    assert D.sample([1.0, math.inf, 3.0, math.inf], 0.9) == (3, 0.5)


def test_u_from_one_on_is_the_last_kept_token():
    """Also where its weight is lost in the running sums."""
    x = np.zeros(200000)
    x[777] = -31.0
    for u in (1.0, 5.0, math.inf):
        assert D.sample(x, u)[0] == 777
        assert D.sample(x, u, min_p=0.5)[0] == 199999
        assert D.sample(x, u, top_k=1000)[0] == 1000  # (777 is the last of all)
        assert D.sample(np.zeros(7), u, top_p=0.5)[0] == 3
    rng = np.random.default_rng(3)
    for _ in range(50):
        x = rng.standard_normal(1000)
        assert D.sample(x, 1.0)[0] == int(np.argmin(x))


def test_moves_read_before_they_write():
    hd = 64
    pool = np.arange(2 * 2 * 2 * 1 * 16 * hd, dtype=np.uint16).reshape(2, 2, 2, 1, 16 * hd)
    k, v = D.tile_places(hd)
    assert sorted(k.ravel()) == sorted(v.ravel()) == list(range(16 * hd))
    new = D.kv_move(pool, hd, [5, 17, -1, 3], [17, 5, 2, 32], [0, 4])
    for c, places in enumerate((k, v)):
        np.testing.assert_array_equal(new[:, 1, c, 0, places[1]], pool[:, 0, c, 0, places[5]])
        np.testing.assert_array_equal(new[:, 0, c, 0, places[5]], pool[:, 1, c, 0, places[1]])
    assert (new != pool).sum() == 2 * 2 * 2 * hd
