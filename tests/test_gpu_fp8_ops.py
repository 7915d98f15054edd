"""The 8-bit feed-forward operators on the GPU against oracle/fp8.py (float64).

Two kinds of products are checked.  With codes that stand for small whole
numbers and powers of two that keep every partial sum within 24 bits, the matrix
cores' sums are exact, so results have to equal the definition bit for bit: that
covers indexes, powers, layouts, slices and row maps.  With normal data the
error bound counts the rounding of the result, half a bf16 step (2^-8), and what
one instruction may cut: of each eight products all but the largest up to 2^-13
of it, 7 * 2^-13 of the sum of magnitudes at most (2^-10 with the fp32 sums).

Codes of 8-bit outputs have to be those of a value within 2^-18 of the
definition's (fp32 evaluation: sums of up to 8192 squares in at most 60 roundings
of 2^-24, halved by the square root, and under ten further roundings).
"""

import numpy as np
import pytest

from oracle import bf16_bits_to_f64, fp8
from paper_2411_03519_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SLACK = 2.0 ** -18


@pytest.fixture(scope="module")
def metro():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2411_03519_amd import metro as m
    return m


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def host(t):
    return t.cpu().numpy()


def bf16(a):
    return synth.f32_to_bf16_bits(np.asarray(a, np.float32))


def bf16_of(t):
    return bf16_bits_to_f64(host(t).view(np.uint16))


def filled(shape, value=0xA5):
    return torch.full(shape, value, dtype=torch.uint8, device="cuda")


def check_rows8(codes, byte, want, slack=SLACK):
    """codes [rows, 128 g], byte [rows, g] are the 8-bit rows of values within `slack` of want [rows, n]."""
    n = want.shape[1]
    q = fp8.grouped(want)
    top = np.max(np.abs(q), axis=2)
    lo, hi = fp8.group_byte(top * (1 - slack)), fp8.group_byte(top * (1 + slack))
    byte = byte.astype(np.int64)
    assert np.all((byte >= lo) & (byte <= hi))
    power = 2.0 ** (byte[:, :, None] - 127.0)
    got = fp8.CODE_VALUES[codes].reshape(q.shape)

    def rounded(v):
        return fp8.CODE_VALUES[fp8.e4m3_code(np.clip(v / power, -448, 448))]

    a, b = rounded(q * (1 - slack)), rounded(q * (1 + slack))
    assert np.all((got >= np.minimum(a, b)) & (got <= np.maximum(a, b)))
    if n % 128:
        assert not np.any(codes[:, n:] & 0x7F)


def whole_rows(rng, rows, K, spread=3):
    """Codes of whole numbers within +-3 and bytes within `spread` powers: sums of K <= 8192 products stay within 24 bits."""
    v = rng.integers(-3, 4, (rows, K)).astype(np.float64)
    return fp8.e4m3_code(v), rng.integers(127, 127 + spread, (rows, K // 128)).astype(np.uint8)


def normal_rows(rng, rows, K, std=1.0):
    return fp8.quantise(rng.normal(size=(rows, K)).astype(np.float32) * std)


def padded(byte, fill=0xFF):
    """Bytes as rows of a multiple of four; the filling is not read (a NaN power would show)."""
    out = np.full((byte.shape[0], -(-byte.shape[1] // 4) * 4), fill, np.uint8)
    out[:, :byte.shape[1]] = byte
    return out


class Operands:
    """X and W of a product (by experts: E matrices W), on the host and on the device."""

    def __init__(self, seed, M, N, K, exact, E=1):
        rng = np.random.default_rng([seed, M, N, K, E])
        self.x = whole_rows(rng, M, K) if exact else normal_rows(rng, M, K)
        self.w = [whole_rows(rng, N, K) if exact else normal_rows(rng, N, K, 0.02) for _ in range(E)]
        self.xv = fp8.values(*self.x)
        self.wv = [fp8.values(*w) for w in self.w]
        self.X, self.xs = dev(self.x[0]), dev(padded(self.x[1]))
        self.W = dev(np.concatenate([fp8.packed_codes(w[0]) for w in self.w]))
        self.ws = dev(np.concatenate([fp8.packed_bytes(w[1], 0xFF) for w in self.w]))


def workspace(M, N, slices=8):
    return torch.full((slices * M * N,), float("nan"), device="cuda") if slices else None


def check_bf16_product(got, y, bound_sum, exact):
    if exact:
        np.testing.assert_array_equal(got, bf16_bits_to_f64(bf16(y)))
    else:
        assert np.all(np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -10 * bound_sum)
        assert np.linalg.norm(got - y) <= 3e-3 * np.linalg.norm(y)


# --- packing -----------------------------------------------------------------


@pytest.mark.parametrize("N,K,ld,Kp", [(16, 128, 128, 128), (48, 200, 208, 256), (96, 687, 700, 768), (32, 1, 1, 128)])
def test_pack_weight_codes_powers_and_layout(metro, N, K, ld, Kp):
    rng = np.random.default_rng(N + K)
    W = bf16(rng.normal(size=(N, ld)) * 2.0 ** rng.integers(-30, 30, (N, 1)))
    W[3, :] = 0
    out, scale = filled((N * Kp,)), filled((N * (-(-Kp // 512) * 4),))
    metro.op_pack_weight_fp8(dev(W), ld, N, K, Kp, out, scale)
    full = np.zeros((N, Kp))
    full[:, :K] = bf16_bits_to_f64(W)[:, :K]
    codes, byte = fp8.quantise(full)
    np.testing.assert_array_equal(host(out), fp8.packed_codes(codes))
    np.testing.assert_array_equal(host(scale), fp8.packed_bytes(byte))


def test_pack_weight_infinities_and_nans(metro):
    W = np.zeros((16, 128), np.uint16)
    W[:, 5] = bf16(np.ones(16))
    W[1, 9], W[2, 9], W[3, 9] = 0x7F80, 0xFF80, 0x7FC0
    out, scale = filled((16 * 128,)), filled((16 * 4,))
    metro.op_pack_weight_fp8(dev(W), 128, 16, 128, 128, out, scale)
    codes = np.empty((16, 128), np.uint8)
    at = fp8.packed_codes(np.arange(128, dtype=np.uint8)[None].repeat(16, 0))
    rows = np.arange(2048) % 256 // 16
    codes[rows, at] = host(out)
    assert (codes[1:4, 9] & 0x7F == 0x7F).all() and (codes[0, 9], codes[0, 5]) == (0, 0x7E - 0x0E + 0x08)
    byte = host(scale).reshape(16, 4)[:, 0]
    assert byte.tolist() == [119, 247, 247, 119] + [119] * 12


def test_groups_of_nothing_but_nans_have_the_least_power(metro):
    W = np.full((16, 256), 0x7FC0, np.uint16)
    W[:, :128] = bf16(np.ones((16, 128)))
    out, scale = filled((16 * 256,)), filled((16 * 4,))
    metro.op_pack_weight_fp8(dev(W), 256, 16, 256, 256, out, scale)
    assert (host(out)[2048:] & 0x7F == 0x7F).all() and host(scale).reshape(16, 4)[:, :2].tolist() == [[119, 1]] * 16
    x = np.ones((2, 200), np.float32)
    x[1, 7] = np.nan
    h, hs = filled((2, 256)), filled((2, 4))
    metro.op_rmsnorm_fp8(dev(x), dev(bf16(np.ones(200))), 0.0, h, hs, 2, 200)
    assert (host(h)[1, :200] & 0x7F == 0x7F).all() and not host(h)[:, 200:].any()
    assert host(hs)[:, :2].tolist() == [[119, 119], [1, 1]]


# --- norm --------------------------------------------------------------------


@pytest.mark.parametrize("rows,d", [(1, 4), (1, 4096), (3, 128), (5, 132), (7, 688), (2, 1000), (4, 5120), (3, 8192), (300, 256)])
@pytest.mark.parametrize("delta,b16", [(False, False), (True, False), (True, True)])
def test_rmsnorm_rows(metro, rows, d, delta, b16):
    rng = np.random.default_rng([rows, d])
    x = (rng.normal(size=(rows, d)) * 2.0 ** rng.integers(-8, 9, (rows, 1))).astype(np.float32)
    dl = bf16(rng.normal(size=(rows, d)))
    gain = bf16(1 + 0.1 * rng.normal(size=d))
    D, G = -(-d // 128) * 128, -(-d // 128)
    L = -(-G // 4) * 4
    h, hs = filled((rows, D)), filled((rows, L))
    xo = torch.full((rows, d), float("nan"), device="cuda") if delta else None
    h16 = torch.zeros(rows, d, dtype=torch.int16, device="cuda") if b16 else None
    metro.op_rmsnorm_fp8(dev(x), dev(gain), 1e-5, h, hs, rows, d, delta=dev(dl) if delta else None, x_out=xo, h_bf16=h16)
    if delta:
        x = x + bf16_bits_to_f64(dl).astype(np.float32)
        np.testing.assert_array_equal(host(xo), x)
    v = fp8.rms_norm(x, bf16_bits_to_f64(gain), 1e-5)
    check_rows8(host(h), host(hs)[:, :G], v)
    assert (host(hs)[:, G:] == 0xA5).all()
    if b16:
        assert np.all(np.abs(bf16_of(h16) - v) <= (2.0 ** -8 + SLACK) * np.abs(v))


@pytest.mark.parametrize("d", [64, 260, 516, 1028, 2048, 2052, 4100])
def test_rmsnorm_rows_of_every_number_of_threads(metro, d):
    rng = np.random.default_rng(d)
    x, gain = rng.normal(size=(3, d)).astype(np.float32), bf16(1 + 0.1 * rng.normal(size=d))
    G = -(-d // 128)
    h, hs = filled((3, 128 * G)), filled((3, -(-G // 4) * 4))
    metro.op_rmsnorm_fp8(dev(x), dev(gain), 1e-5, h, hs, 3, d)
    check_rows8(host(h), host(hs)[:, :G], fp8.rms_norm(x, bf16_bits_to_f64(gain), 1e-5))


def test_rmsnorm_strides_and_sum_in_place(metro):
    rows, d, ldx, ldd, ldb, ldh, lds = 5, 388, 400, 404, 392, 528, 9
    rng = np.random.default_rng(3)
    x = rng.normal(size=(rows, ldx)).astype(np.float32)
    dl, gain = bf16(rng.normal(size=(rows, ldd))), bf16(np.ones(d))
    X, h, hs = dev(x), filled((rows, ldh)), filled((rows, lds))
    h16 = torch.full((rows, ldb), 77, dtype=torch.int16, device="cuda")
    metro.op_rmsnorm_fp8(X, dev(gain), 1e-6, h, hs, rows, d, delta=dev(dl), x_out=X, h_bf16=h16, ldx=ldx, ldd=ldd,
                         ldh_bf16=ldb, ldh=ldh, lds=lds)
    want = x.copy()
    want[:, :d] += bf16_bits_to_f64(dl)[:, :d].astype(np.float32)
    np.testing.assert_array_equal(host(X), want)
    v = fp8.rms_norm(want[:, :d], np.ones(d), 1e-6)
    check_rows8(host(h)[:, :512], host(hs)[:, :4], v)
    assert (host(h)[:, 512:] == 0xA5).all() and (host(hs)[:, 4:] == 0xA5).all() and (host(h16)[:, d:] == 77).all()


def test_rmsnorm_zero_infinite_and_nan_rows(metro):
    d = 256
    x = np.ones((4, d), np.float32)
    x[0], x[1, 7], x[2, 200] = 0, np.nan, np.inf
    h, hs = filled((4, d)), filled((4, 4))
    metro.op_rmsnorm_fp8(dev(x), dev(bf16(np.ones(d))), 1e-5, h, hs, 4, d)
    h, hs = host(h), host(hs)[:, :2]
    assert not h[0].any() and hs[0].tolist() == [1, 1]
    assert (h[1] & 0x7F == 0x7F).all()
    assert h[2, 200] & 0x7F == 0x7F and not np.delete(h[2], 200).any()  # 1 / inf = 0, inf / inf = NaN
    check_rows8(h[3:], hs[3:], fp8.rms_norm(x[3:], np.ones(d), 1e-5))


def test_rmsnorm_without_rows_touches_nothing(metro):
    h, hs = filled((1, 128)), filled((1, 4))
    metro.op_rmsnorm_fp8(torch.zeros(1, 128, device="cuda"), dev(bf16(np.ones(128))), 1e-5, h, hs, 0, 128)
    assert (host(h) == 0xA5).all() and (host(hs) == 0xA5).all()


# --- products ------------------------------------------------------------------


SHAPES = [(1, 32, 128), (1, 4096, 4096), (7, 96, 384), (16, 256, 512), (17, 288, 640), (25, 1376, 256), (33, 512, 1152),
          (64, 2080, 1408), (65, 256, 768), (100, 544, 128), (128, 1056, 2048), (200, 768, 1024), (257, 320, 640),
          (300, 1376, 256), (513, 800, 896), (1001, 512, 384), (1, 32, 4096), (129, 6144, 512), (700, 2048, 256)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("ws", [0, 8])
@pytest.mark.parametrize("exact", [True, False])
def test_product_to_bf16_rows(metro, M, N, K, ws, exact):
    o = Operands(1, M, N, K, exact)
    out = torch.full((M + 1, N), 77, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8(o.X, o.xs, o.W, o.ws, M, N, K, metro.EPI_FP8_BF16, out, workspace=workspace(M, N, ws))
    assert (host(out)[M] == 77).all()
    check_bf16_product(bf16_of(out[:M]), o.xv @ o.wv[0].T, np.abs(o.xv) @ np.abs(o.wv[0].T), exact)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("ws", [0, 8])
def test_product_with_swiglu_to_8_bit_rows(metro, M, N, K, ws):
    # (whole numbers: gate and up are exact, so only the activation's fp32 evaluation is left)
    o = Operands(2, M, N, K, True)
    F = N // 2
    G = -(-F // 128)
    out, scale = filled((M + 1, G * 128)), filled((M + 1, -(-G // 4) * 4))
    # powers that bring gates to a few units: some features live, some off
    o.ws -= 7
    y = (o.xv @ o.wv[0].T) * 2.0 ** -7
    metro.op_gemm_fp8(o.X, o.xs, o.W, o.ws, M, N, K, metro.EPI_FP8_SWIGLU, out, out_scale=scale,
                      workspace=workspace(M, N, ws))
    check_rows8(host(out)[:M], host(scale)[:M, :G], fp8.swiglu_rows(y), slack=2.0 ** -17)
    assert (host(out)[M] == 0xA5).all() and (host(scale)[M] == 0xA5).all() and (host(scale)[:, G:] == 0xA5).all()


def test_product_takes_the_powers_of_its_own_blocks(metro):
    """Every block of 128 has another power on both sides, from 2^-40 to 2^40, so that one taken from a wrong block, row or
    half shows; one code per block, at another column each, keeps the sums exact."""
    M, N, K = 35, 64, 1664
    rng = np.random.default_rng(5)
    xc, wc = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    B = K // 128
    keep = rng.integers(0, B, (M, N))
    wc[:] = fp8.e4m3_code(rng.integers(1, 4, (N, K)).astype(float))
    xb, wb = rng.integers(87, 168, (M, B)).astype(np.uint8), rng.integers(87, 168, (N, B)).astype(np.uint8)
    for m in range(M):  # one block of X lives in each row
        b = keep[m, 0]
        xc[m, b * 128 + rng.integers(0, 128)] = fp8.e4m3_code(np.array([3.0]))[0]
    out = torch.zeros(M, N, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8(dev(xc), dev(padded(xb)), dev(fp8.packed_codes(wc)), dev(fp8.packed_bytes(wb, 0xFF)), M, N, K,
                      metro.EPI_FP8_BF16, out)
    y = fp8.values(xc, xb) @ fp8.values(wc, wb).T
    np.testing.assert_array_equal(bf16_of(out), bf16_bits_to_f64(bf16(y)))


@pytest.mark.parametrize("M,N,K", [(5, 160, 384), (70, 288, 256), (260, 544, 640)])
def test_product_strides(metro, M, N, K):
    o = Operands(4, M, N, K, True)
    ldx, ldxs, ldo = K + 48, 4 * (K // 512 + 3), N + 12
    x = np.full((M, ldx), 0x7F, np.uint8)
    x[:, :K] = o.x[0]
    xs = np.full((M, ldxs), 0xFF, np.uint8)
    xs[:, :K // 128] = o.x[1]
    out = torch.full((M, ldo), 77, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8(dev(x), dev(xs), o.W, o.ws, M, N, K, metro.EPI_FP8_BF16, out, ldx=ldx, ldxs=ldxs, ldo=ldo)
    assert (host(out)[:, N:] == 77).all()
    check_bf16_product(bf16_of(out)[:, :N], o.xv @ o.wv[0].T, None, True)
    F, G = N // 2, -(-(N // 2) // 128)
    ldo, ldos = G * 128 + 32, G + 3
    out, scale = filled((M, ldo)), filled((M, ldos))
    o.ws -= 7
    metro.op_gemm_fp8(dev(x), dev(xs), o.W, o.ws, M, N, K, metro.EPI_FP8_SWIGLU, out, out_scale=scale, ldx=ldx, ldxs=ldxs,
                      ldo=ldo, ldos=ldos, workspace=workspace(M, N))
    assert (host(out)[:, G * 128:] == 0xA5).all() and (host(scale)[:, G:] == 0xA5).all()
    check_rows8(host(out)[:, :G * 128], host(scale)[:, :G], fp8.swiglu_rows((o.xv @ o.wv[0].T) / 128), slack=2.0 ** -17)


def test_product_of_nan_rows_stays_in_its_row(metro):
    M, N, K = 40, 288, 256
    o = Operands(6, M, N, K, True)
    x = o.x[0].copy()
    x[11, 130] = 0x7F
    out = torch.zeros(M, N, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8(dev(x), o.xs, o.W, o.ws, M, N, K, metro.EPI_FP8_BF16, out)
    got, y = bf16_of(out), bf16_bits_to_f64(bf16(o.xv @ o.wv[0].T))
    assert np.isnan(got[11]).all()
    np.testing.assert_array_equal(np.delete(got, 11, 0), np.delete(y, 11, 0))


@pytest.mark.parametrize("M,ws", [(5, 0), (40, 0), (40, 8), (150, 0), (700, 0)])
def test_swiglu_of_nan_and_infinite_rows_stays_in_its_rows(metro, M, ws):
    N, K = 544, 512
    o = Operands(7, M, N, K, False)
    x, xs, F = o.x[0].copy(), o.xs.clone(), N // 2
    outs = []
    for bad in (False, True):
        if bad:
            x[1, 300] = 0x7F  # a NaN code
            x[3], xs[3, :4] = 0x7E, 254  # 448 * 2^127 in each column: infinite sums
        out, scale = filled((M, 384)), filled((M, 4))
        metro.op_gemm_fp8(dev(x), xs, o.W, o.ws, M, N, K, metro.EPI_FP8_SWIGLU, out, out_scale=scale, workspace=workspace(M, N, ws))
        outs.append((host(out), host(scale)[:, :3]))
    (codes, byte), (codes_bad, byte_bad) = outs
    assert (codes_bad[1, :F] & 0x7F == 0x7F).all() and (byte_bad[1] == 1).all()
    # infinite where the weights' sum is not next to 0; an infinite factor makes an infinity or a NaN
    infinite = (np.abs(o.wv[0].sum(1)) > 0.05).reshape(N // 16, 2, 8).any(1).reshape(F)
    assert infinite.mean() > 0.9 and (codes_bad[3, :F][infinite] & 0x7F == 0x7F).all()
    for rest in (codes_bad, codes), (byte_bad, byte):
        np.testing.assert_array_equal(*[np.delete(v, [1, 3], 0) for v in rest])


def test_product_repeats_bit_for_bit(metro):
    for M, N, K in ((25, 1376, 2048), (301, 544, 1024)):
        o = Operands(7, M, N, K, False)
        outs = []
        for _ in range(4):
            out = torch.zeros(M, N, dtype=torch.int16, device="cuda")
            metro.op_gemm_fp8(o.X, o.xs, o.W, o.ws, M, N, K, metro.EPI_FP8_BF16, out, workspace=workspace(M, N))
            outs.append(host(out))
        for other in outs[1:]:
            np.testing.assert_array_equal(outs[0], other)


# --- routing -------------------------------------------------------------------


def run_route(metro, z, k, bias=None, **kw):
    T, E = z.shape
    i32 = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")  # noqa: E731
    experts, offsets, src, slot = i32(T, k), i32(E + 1), i32(T * k), i32(T, k)
    w = torch.full((T, k), -77.0, device="cuda")
    ws = i32(-(-T // 64) * E)
    metro.op_route(dev(z.astype(np.float32)), T, E, k, experts, w, offsets, src, slot,
                   bias=None if bias is None else dev(np.asarray(bias, np.float32)), workspace=ws, **kw)
    return [host(t) for t in (experts, w, offsets, src, slot)]


def check_route(metro, z, k, bias=None, scoring=0, n_groups=1, top_groups=1, renormalise=True, scale=1.0):
    got = run_route(metro, z, k, bias, scoring=scoring, n_groups=n_groups, top_groups=top_groups, renormalise=renormalise,
                    scale=scale)
    want = fp8.route(z.astype(np.float32), k, None if bias is None else np.asarray(bias, np.float32), bool(scoring), n_groups,
                     top_groups, renormalise, scale)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_allclose(got[1], want[1], rtol=2.0 ** -23, atol=1e-45)  # one rounding to fp32, of fp64 values
    for a, b in zip(got[2:], want[2:]):
        np.testing.assert_array_equal(a, b)
    return got


@pytest.mark.parametrize("T", [1, 25, 63, 64, 65, 200, 1000])
@pytest.mark.parametrize("E,k,groups,top", [(1, 1, 1, 1), (8, 2, 1, 1), (8, 2, 4, 2), (13, 3, 1, 1), (16, 16, 4, 4), (32, 4, 8, 3),
                                            (60, 6, 1, 1), (64, 8, 64, 9), (128, 8, 8, 4), (256, 8, 8, 4), (500, 7, 5, 1)])
def test_route_choices_weights_and_order(metro, T, E, k, groups, top):
    rng = np.random.default_rng([T, E, k])
    z = rng.normal(size=(T, E)) * 2
    scoring = (T + E) % 2
    check_route(metro, z, k, rng.normal(size=E) * 0.1 if T % 2 else None, scoring, groups, top, T % 3 > 0, 1.0 + (T % 2) * 1.5)


def test_route_ties_go_to_the_lowest_index(metro):
    z = np.zeros((130, 64))
    z[::3, 40] = 1
    z[1::3] = np.tile([1.0, 0.0], 32)
    check_route(metro, z, 5)
    check_route(metro, z, 5, scoring=1, n_groups=8, top_groups=2)


@pytest.mark.parametrize("T", [3, 9, 64, 150])
@pytest.mark.parametrize("E,k,groups,top", [(16, 2, 16, 5), (24, 3, 12, 4), (32, 6, 32, 7), (48, 5, 24, 9), (64, 6, 32, 5), (128, 8, 64, 20),
                                            (130, 8, 26, 3), (256, 8, 64, 6), (512, 9, 64, 9)])
def test_route_more_groups_than_lanes_and_equal_scores(metro, T, E, k, groups, top):
    rng = np.random.default_rng([T, E, groups])
    check_route(metro, rng.integers(0, 4, (T, E)) / 2.0, k, None, T % 2, groups, top)
    z = rng.integers(0, 2, (T, E)) + 2.0 ** -22 * rng.integers(0, 3, (T, E))  # mostly apart in the lower bits alone
    check_route(metro, z, k, None, 1 - T % 2, groups, top)


@pytest.mark.parametrize("T", [5, 70])
@pytest.mark.parametrize("scoring", [0, 1])
def test_route_masked_infinite_and_nan_logits(metro, T, scoring):
    rng = np.random.default_rng(T)
    z = rng.normal(size=(T, 16))
    z[0] = -np.inf
    z[1, 3:] = -np.inf
    z[2, 5] = np.nan
    z[3] = np.nan
    z[4, :15] = np.finfo(np.float32).min
    with np.errstate(all="ignore"):
        for groups, top in ((1, 1), (4, 2)):
            check_route(metro, z, 4, scoring=scoring, n_groups=groups, top_groups=top)
            check_route(metro, z, 4, scoring=scoring, n_groups=groups, top_groups=top, renormalise=False)
        bias = np.zeros(16)
        bias[[0, 7]] = -np.inf
        bias[9] = np.nan
        got = check_route(metro, z, 4, bias, scoring=scoring)
        assert not np.isin(got[0][5:], [0, 7, 9]).any()


def test_route_logits_of_a_wider_product(metro):
    z = np.random.default_rng(2).normal(size=(90, 32)).astype(np.float32)
    Z = dev(z)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    experts, offsets, src, slot, w = i32(90, 2), i32(9), i32(180), i32(90, 2), torch.zeros(90, 2, device="cuda")
    metro.op_route(Z, 90, 8, 2, experts, w, offsets, src, slot, ldl=32, workspace=i32(2 * 8))
    want = fp8.route(z[:, :8], 2)
    np.testing.assert_array_equal(host(experts), want[0])
    np.testing.assert_array_equal(host(src), want[3])


def test_route_without_tokens_has_empty_experts(metro):
    got = run_route(metro, np.zeros((0, 8)), 2)
    assert got[2].tolist() == [0] * 9


# --- experts ---------------------------------------------------------------------


def offsets_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


EXPERTS = [([3, 0, 5, 1], 160, 256), ([0, 0, 0, 0], 160, 256), ([0, 70, 0], 288, 384), ([17, 16, 15, 1, 0, 33], 96, 128),
           ([130, 1, 260, 0, 64], 544, 256), ([1] * 70, 64, 128), ([300, 300], 512, 1152), ([2, 700, 40], 800, 640)]


@pytest.mark.parametrize("counts,N,K", EXPERTS)
@pytest.mark.parametrize("gathered", [True, False])
@pytest.mark.parametrize("ws", [0, 8])
def test_experts_product(metro, counts, N, K, gathered, ws):
    E, R, spare = len(counts), sum(counts), 3  # slots behind the last expert's
    T = 50 if gathered else R + spare
    o = Operands(8, T, N, K, True, E)
    offsets = offsets_of(counts)
    rng = np.random.default_rng(R)
    src = rng.integers(0, T, R + spare).astype(np.int32) if gathered else np.arange(R + spare, dtype=np.int32)
    y = np.zeros((R, N))
    for e in range(E):
        y[offsets[e]:offsets[e + 1]] = o.xv[src[offsets[e]:offsets[e + 1]]] @ o.wv[e].T
    S = dev(src) if gathered else None
    out = torch.full((R + spare, N), 77, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8_experts(o.X, o.xs, T, S, dev(offsets), E, R + spare, o.W, o.ws, N, K, metro.EPI_FP8_BF16, out,
                              workspace=workspace(R + spare, N, ws))
    assert (host(out)[R:] == 77).all()
    check_bf16_product(bf16_of(out[:R]), y, None, True)
    G = -(-(N // 2) // 128)
    out, scale = filled((R + spare, G * 128)), filled((R + spare, -(-G // 4) * 4))
    o.ws -= 7
    metro.op_gemm_fp8_experts(o.X, o.xs, T, S, dev(offsets), E, R + spare, o.W, o.ws, N, K, metro.EPI_FP8_SWIGLU, out,
                              out_scale=scale, workspace=workspace(R + spare, N, ws))
    assert (host(out)[R:] == 0xA5).all() and (host(scale)[R:] == 0xA5).all()
    check_rows8(host(out)[:R], host(scale)[:R, :G], fp8.swiglu_rows(y / 128), slack=2.0 ** -17)


def test_experts_indexes_are_held_in_range(metro):
    """Rows of X and offsets outside their ranges reach other valid rows, never memory outside the buffers."""
    T, N, K, E, R = 20, 64, 128, 3, 40
    o = Operands(9, T, N, K, True, E)
    src = np.array([-5, T, 1 << 30] + [3] * (R - 3), np.int32)
    out = torch.full((R + 1, N), 77, dtype=torch.int16, device="cuda")
    metro.op_gemm_fp8_experts(o.X, o.xs, T, dev(src), dev(np.array([0, 10, 5, 1000], np.int32)), E, R, o.W, o.ws, N, K,
                              metro.EPI_FP8_BF16, out)
    got = bf16_of(out)
    assert (host(out)[R] == 77).all()
    np.testing.assert_array_equal(got[3:5], bf16_bits_to_f64(bf16(o.xv[[3, 3]] @ o.wv[0].T)))
    np.testing.assert_array_equal(got[10:R], bf16_bits_to_f64(bf16(o.xv[[3] * (R - 10)] @ o.wv[2].T)))


def test_one_expert_is_the_dense_product(metro):
    for M, N, K in ((25, 544, 512), (300, 288, 384)):
        o = Operands(10, M, N, K, False)
        a, b = (torch.zeros(M, N, dtype=torch.int16, device="cuda") for _ in range(2))
        metro.op_gemm_fp8(o.X, o.xs, o.W, o.ws, M, N, K, metro.EPI_FP8_BF16, a)
        metro.op_gemm_fp8_experts(o.X, o.xs, M, None, dev(offsets_of([M])), 1, M, o.W, o.ws, N, K, metro.EPI_FP8_BF16, b)
        A, B = bf16_of(a), bf16_of(b)
        # (kernels may sum k in another order: a step of bf16 apart at most)
        assert np.all(np.abs(A - B) <= 2.0 ** -7 * np.abs(A) + 2.0 ** -10 * (np.abs(o.xv) @ np.abs(o.wv[0].T)))


# --- combine ---------------------------------------------------------------------


@pytest.mark.parametrize("T,k,d", [(1, 1, 8), (25, 2, 4096), (7, 3, 1000), (300, 8, 256), (65, 2, 8200)])
@pytest.mark.parametrize("resid", [True, False])
def test_combine(metro, T, k, d, resid):
    rng = np.random.default_rng([T, k, d])
    R = T * k
    y, w = bf16(rng.normal(size=(R, d))), rng.random((T, k)).astype(np.float32)
    slot = rng.permutation(R).reshape(T, k).astype(np.int32)
    if T > 1:
        slot[1] = -1
        slot[0, 0] = R
    x = rng.normal(size=(T, d)).astype(np.float32)
    out = torch.full((T, d), float("nan"), device="cuda")
    metro.op_combine_experts(dev(y), R, dev(w), dev(slot), T, k, d, out, resid=dev(x) if resid else None)
    yv = bf16_bits_to_f64(y)
    want = fp8.combine(yv, w, slot, x if resid else None)
    size = fp8.combine(np.abs(yv), w, slot, np.abs(x) if resid else None)
    assert np.all(np.abs(host(out) - want) <= (k + 1) * 2.0 ** -24 * size)


def test_combine_strides_and_in_place(metro):
    T, k, d, ldy, ldo = 9, 2, 40, 48, 44
    rng = np.random.default_rng(1)
    y, w = bf16(rng.normal(size=(T * k, ldy))), rng.random((T, k)).astype(np.float32)
    slot = rng.permutation(T * k).reshape(T, k).astype(np.int32)
    x = rng.normal(size=(T, ldo)).astype(np.float32)
    X = dev(x)
    metro.op_combine_experts(dev(y), T * k, dev(w), dev(slot), T, k, d, X, resid=X, ldy=ldy, ldo=ldo)
    want = fp8.combine(bf16_bits_to_f64(y)[:, :d], w, slot, x[:, :d])
    np.testing.assert_allclose(host(X)[:, :d], want, rtol=0, atol=3 * 2.0 ** -24 * 16)
    np.testing.assert_array_equal(host(X)[:, d:], x[:, d:])


# --- together ----------------------------------------------------------------------


class Block:
    """A feed-forward block by experts as a serving loop runs it: norm with the pending residual rows, router product, routing,
    gate and up, down, weighted sum.  Buffers for up to `cap` tokens; run() only launches."""

    d, F, E, k = 256, 688, 8, 2

    def __init__(self, metro, cap, seed=0):
        self.m, self.cap = metro, cap
        d, F, E, k = self.d, self.F, self.E, self.k
        self.Fp = -(-F // 128) * 128
        rng = np.random.default_rng(seed)
        self.gain = bf16(1 + 0.1 * rng.normal(size=d))
        router = np.zeros((32, d), np.uint16)
        router[:E] = bf16(rng.normal(size=(E, d)) * 0.1)
        self.router = router
        up = bf16(rng.normal(size=(E, 2 * F, d)) * 0.08)
        down = bf16(rng.normal(size=(E, d, F)) * 0.05)
        q = [fp8.quantise(bf16_bits_to_f64(w)) for w in up]
        self.up = [fp8.values(*w) for w in q]
        q = [fp8.quantise(bf16_bits_to_f64(w)) for w in down]
        self.down = [fp8.values(*w)[:, :F] for w in q]
        u8 = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        i16 = lambda *s: torch.zeros(s, dtype=torch.int16, device="cuda")  # noqa: E731
        self.W1, self.s1, self.W2, self.s2 = u8(E * 2 * F * d), u8(E * 2 * F * 4), u8(E * d * self.Fp), u8(E * d * 8)
        for e in range(E):
            metro.op_pack_weight_fp8(dev(up[e]), d, 2 * F, d, d, self.W1[e * 2 * F * d:], self.s1[e * 2 * F * 4:])
            metro.op_pack_weight_fp8(dev(down[e]), F, d, F, self.Fp, self.W2[e * d * self.Fp:], self.s2[e * d * 8:])
        self.Wr = i16(32 * d)
        metro.op_pack_weight(dev(router), d, 32, d, d, self.Wr)
        self.g = dev(self.gain)
        R = cap * k
        self.x, self.delta = torch.zeros(cap, d, device="cuda"), i16(cap, d)
        self.h, self.hs, self.h16 = u8(cap * d).view(cap, d), u8(cap * 4).view(cap, 4), i16(cap, d)
        self.logits = torch.zeros(cap, 32, device="cuda")
        self.experts, self.offsets, self.src, self.slot = i32(cap, k), i32(E + 1), i32(R), i32(cap, k)
        self.w, self.rws = torch.zeros(cap, k, device="cuda"), i32(-(-cap // 64) * E)
        self.a, self.as_, self.y = u8(R * self.Fp).view(R, self.Fp), u8(R * 8).view(R, 8), i16(R, d)
        self.ws = torch.zeros(8 * R * 2 * F, device="cuda")
        self.out = torch.zeros(cap, d, device="cuda")

    def run(self, T):
        m, d, F, E, k, R = self.m, self.d, self.F, self.E, self.k, T * self.k
        m.op_rmsnorm_fp8(self.x, self.g, 1e-5, self.h, self.hs, T, d, delta=self.delta, x_out=self.x, h_bf16=self.h16)
        m.op_gemm(self.h16, self.Wr, T, 32, d, m.EPI_STORE_F32, self.logits, 32)
        m.op_route(self.logits, T, E, k, self.experts, self.w, self.offsets, self.src, self.slot, ldl=32, workspace=self.rws)
        m.op_gemm_fp8_experts(self.h, self.hs, T, self.src, self.offsets, E, R, self.W1, self.s1, 2 * F, d, m.EPI_FP8_SWIGLU,
                              self.a, out_scale=self.as_, workspace=self.ws)
        m.op_gemm_fp8_experts(self.a, self.as_, R, None, self.offsets, E, R, self.W2, self.s2, d, self.Fp, m.EPI_FP8_BF16,
                              self.y, workspace=self.ws)
        m.op_combine_experts(self.y, R, self.w, self.slot, T, k, d, self.out, resid=self.x)

    def set_inputs(self, T, seed):
        rng = np.random.default_rng([T, seed])
        x, delta = rng.normal(size=(T, self.d)).astype(np.float32), bf16(rng.normal(size=(T, self.d)) * 0.3)
        self.x[:T] = dev(x)
        self.delta[:T] = dev(delta)
        return x + bf16_bits_to_f64(delta).astype(np.float32)

    def check(self, T, x):
        """Each step against its definition on the inputs that the step had."""
        np.testing.assert_array_equal(host(self.x[:T]), x)
        v = fp8.rms_norm(x, bf16_bits_to_f64(self.gain), 1e-5)
        check_rows8(host(self.h[:T]), host(self.hs[:T])[:, :2], v)
        want = fp8.route(host(self.logits[:T])[:, :self.E], self.k)
        np.testing.assert_array_equal(host(self.experts[:T]), want[0])
        np.testing.assert_array_equal(host(self.src)[:T * self.k], want[3])
        hv = fp8.values(host(self.h[:T]), host(self.hs[:T]))
        av = fp8.values(host(self.a[:T * self.k]), host(self.as_[:T * self.k]))[:, :self.F]
        y = bf16_of(self.y[:T * self.k])
        for e in range(self.E):
            lo, hi = want[2][e], want[2][e + 1]
            act = fp8.swiglu_rows(hv[want[3][lo:hi]] @ self.up[e].T)
            # half a step of e4m3 (2^-4), and the products' 2^-10 of their magnitudes through the activation
            assert np.linalg.norm(av[lo:hi] - act) <= 0.04 * np.linalg.norm(act)
            z = av[lo:hi] @ self.down[e].T
            assert np.all(np.abs(y[lo:hi] - z) <= 2.0 ** -8 * np.abs(z) + 2.0 ** -10 * (np.abs(av[lo:hi]) @ np.abs(self.down[e].T)))
        got = host(self.out[:T])
        np.testing.assert_allclose(got, fp8.combine(y, host(self.w[:T]), host(self.slot[:T]), x), rtol=0, atol=2e-6)
        # and the block as a whole against float64 without any 8-bit rounding of its activations: e4m3's half steps in two
        # places, each spread evenly over +-2^-4 (rms 2^-4 / sqrt(3) = 0.036 at most), sqrt(2) of them and some room
        full = x.astype(np.float64).copy()
        for e in range(self.E):
            lo, hi = want[2][e], want[2][e + 1]
            rows = want[3][lo:hi]
            f = fp8.swiglu_rows(v[rows] @ self.up[e].T) @ self.down[e].T
            for i, t in enumerate(rows):
                full[t] += host(self.w[t])[list(want[0][t]).index(e)] * f[i]
        assert np.linalg.norm(got - full) <= 0.07 * np.linalg.norm(full - x)


@pytest.mark.parametrize("T", [1, 25, 300])
def test_feed_forward_block_by_experts(metro, T):
    b = Block(metro, T)
    x = b.set_inputs(T, 1)
    b.run(T)
    b.check(T, x)


def test_block_on_another_stream_and_replayed_from_graphs(metro):
    """Two captured blocks of their own buffers, replayed in turn with eager work of other sizes between them."""
    s = torch.cuda.Stream()
    blocks = [Block(metro, 100, 1), Block(metro, 100, 2)]
    eager = Block(metro, 130, 3)
    graphs = []
    with torch.cuda.stream(s):
        for b in blocks:
            b.run(100)  # (kernels loaded)
        s.synchronize()
        for b in blocks:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                b.run(100)
            graphs.append(g)
        for turn in range(3):
            xs = [b.set_inputs(100, 10 * turn + i) for i, b in enumerate(blocks)]
            x = eager.set_inputs(130 - turn, turn)
            for g in graphs:
                g.replay()
            eager.run(130 - turn)
            s.synchronize()
            for b, bx in zip(blocks, xs):
                b.check(100, bx)
            eager.check(130 - turn, x)


def test_dense_feed_forward_block(metro):
    d, F, M = 256, 688, 77
    Fp = 768
    rng = np.random.default_rng(4)
    up, down = bf16(rng.normal(size=(2 * F, d)) * 0.08), bf16(rng.normal(size=(d, F)) * 0.05)
    W1, s1, W2, s2 = filled((2 * F * d,)), filled((2 * F * 4,)), filled((d * Fp,)), filled((d * 8,))
    metro.op_pack_weight_fp8(dev(up), d, 2 * F, d, d, W1, s1)
    metro.op_pack_weight_fp8(dev(down), F, d, F, Fp, W2, s2)
    x, gain = rng.normal(size=(M, d)).astype(np.float32), bf16(np.ones(d))
    h, hs, a, as_ = filled((M, d)), filled((M, 4)), filled((M, Fp)), filled((M, 8))
    y = torch.zeros(M, d, dtype=torch.int16, device="cuda")
    X, xo = dev(x), torch.zeros(M, d, device="cuda")
    metro.op_rmsnorm_fp8(X, dev(gain), 1e-5, h, hs, M, d)
    metro.op_gemm_fp8(h, hs, W1, s1, M, 2 * F, d, metro.EPI_FP8_SWIGLU, a, out_scale=as_, workspace=workspace(M, 2 * F))
    metro.op_gemm_fp8(a, as_, W2, s2, M, d, Fp, metro.EPI_FP8_BF16, y, workspace=workspace(M, d))
    metro.op_rmsnorm_fp8(X, dev(gain), 1e-5, h, hs, M, d, delta=y, x_out=xo)
    v = fp8.rms_norm(x, np.ones(d), 1e-5)
    f = fp8.swiglu_rows(v @ bf16_bits_to_f64(up).T) @ bf16_bits_to_f64(down).T
    got = host(xo) - x
    # rows, weights, activation rows and weights in e4m3: four roundings of rms 0.036 at most
    assert np.linalg.norm(got - f) <= 0.08 * np.linalg.norm(f)
