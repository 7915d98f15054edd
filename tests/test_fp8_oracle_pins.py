"""Pins of the plain definitions of the 8-bit feed-forward operators (oracle/fp8.py):
values worked out by hand, and torch's own e4m3 conversion."""

import numpy as np
import pytest

from oracle import fp8

torch = pytest.importorskip("torch")


def test_code_values_by_hand():
    v = fp8.CODE_VALUES
    assert [v[c] for c in (0x00, 0x01, 0x07, 0x08, 0x38, 0x39, 0x7E)] == [0.0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.0,
                                                                          1.125, 448.0]
    assert v[0xB8] == -1.0 and np.isnan(v[0x7F]) and np.isnan(v[0xFF])


def test_codes_equal_torchs_conversion():
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000),
                        fp8._POSITIVE, -fp8._POSITIVE, (fp8._POSITIVE[1:] + fp8._POSITIVE[:-1]) / 2]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(fp8.e4m3_code(v), want)


@pytest.mark.parametrize("top,byte", [(448.0, 127), (448.00003, 128), (224.0, 126), (1.0, 119), (1.75, 119), (1.7500001, 120),
                                      (0.0, 1), (2.0 ** -140, 1), (3.4028235e38, 247), (np.inf, 247), (448.0 * 2.0 ** -126, 1), (449.0 * 2.0 ** -126, 2)])
def test_group_byte_at_its_borders(top, byte):
    assert fp8.group_byte(np.array([top]))[0] == byte


def test_quantised_values_are_within_half_a_step():
    rng = np.random.default_rng(1)
    v = rng.normal(size=(7, 300)) * 2.0 ** rng.integers(-20, 20, (7, 1))
    codes, byte = fp8.quantise(v)
    assert codes.shape == (7, 384) and byte.shape == (7, 3) and not codes[:, 300:].any()
    got = fp8.values(codes, byte)[:, :300]
    step = np.repeat(2.0 ** (byte.astype(float) - 127), 128, axis=1)[:, :300]
    assert np.all(np.abs(got - v) <= np.maximum(np.abs(v) * 2.0 ** -4, step * 2.0 ** -10))


def test_swiglu_pairs_columns_of_eights():
    y = np.zeros((1, 32))
    y[0, 3], y[0, 11], y[0, 16 + 5], y[0, 24 + 5] = 2.0, 3.0, -1.0, 4.0
    out = fp8.swiglu_rows(y)
    want = np.zeros((1, 16))
    want[0, 3], want[0, 13] = 2.0 / (1 + np.exp(-2.0)) * 3.0, -1.0 / (1 + np.exp(1.0)) * 4.0
    np.testing.assert_allclose(out, want, rtol=1e-15)


def test_route_by_hand():
    logits = np.log([[1, 2, 3, 4], [4, 4, 1, 1], [1, 1, 1, 1.0]])
    experts, w, offsets, src, slot = fp8.route(logits, 2)
    assert experts.tolist() == [[3, 2], [0, 1], [0, 1]]
    np.testing.assert_allclose(w, [[4 / 7, 3 / 7], [0.5, 0.5], [0.5, 0.5]])
    assert offsets.tolist() == [0, 2, 4, 5, 6] and src.tolist() == [1, 2, 1, 2, 0, 0]
    assert slot.tolist() == [[5, 4], [0, 2], [1, 3]]


def test_route_groups_and_bias_by_hand():
    # groups {0, 1}, {2, 3}: sums of sigmoids 0.9 + 0.1 against 0.6 + 0.6: the second stays
    z = np.log(np.array([[0.9, 0.1, 0.6, 0.6]]) / (1 - np.array([[0.9, 0.1, 0.6, 0.6]])))
    experts, w, *_ = fp8.route(z, 2, sigmoid=True, groups=2, top_groups=1, renormalise=False, scale=2.0)
    assert experts.tolist() == [[2, 3]]
    np.testing.assert_allclose(w, [[1.2, 1.2]])
    # a bias moves the choice, not the weight
    experts, w, *_ = fp8.route(z, 1, bias=[0, 1.0, 0, 0], sigmoid=True, renormalise=False)
    assert experts.tolist() == [[1]]
    np.testing.assert_allclose(w, [[0.1]])


def test_route_with_nothing_left():
    z = np.array([[-np.inf] * 4, [np.nan, 1.0, 2.0, 3.0], [-np.inf, -np.inf, 0.0, -np.inf]])
    experts, w, *_ = fp8.route(z, 2)
    assert experts.tolist() == [[0, 1], [0, 1], [2, 0]]
    assert w[0].tolist() == [0, 0] and np.isnan(w[1]).all() and w[2].tolist() == [1, 0]
    experts, w, *_ = fp8.route(z, 2, sigmoid=True, renormalise=False)
    assert experts[1].tolist() == [3, 2]


def test_combine_by_hand():
    y = np.array([[1.0, 2], [3, 4], [5, 6]])
    out = fp8.combine(y, [[0.5, 2.0], [1.0, 1.0]], np.array([[2, 0], [1, -1]]), resid=[[1.0, 1], [0, 0]])
    assert out.tolist() == [[1 + 2.5 + 2, 1 + 3 + 4], [3, 4]]


def test_packed_layout_is_the_headers():
    N, K = 32, 256
    codes = (np.arange(N * K) % 251).astype(np.uint8).reshape(N, K)
    flat = fp8.packed_codes(codes)
    assert flat[0:16].tolist() == codes[0, :16].tolist()          # row 0, columns 0 .. 15
    assert flat[16:32].tolist() == codes[1, :16].tolist()         # row 1
    assert flat[256:272].tolist() == codes[0, 16:32].tolist()     # row 0, columns 16 .. 31
    assert flat[1024:1040].tolist() == codes[0, 64:80].tolist()   # second half of the 128
    assert flat[2048:2064].tolist() == codes[0, 128:144].tolist()
    assert flat[16 * K:16 * K + 16].tolist() == codes[16, :16].tolist()
    b = fp8.packed_bytes(np.arange(N * 2, dtype=np.uint8).reshape(N, 2))
    assert b[:8].tolist() == [0, 1, 127, 127, 2, 3, 127, 127] and b[64:66].tolist() == [32, 33]
