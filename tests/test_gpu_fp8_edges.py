"""The 8-bit rows at their edges."""

import numpy as np
import pytest

from oracle import fp8
from tests.test_gpu_fp8_ops import check_rows8, dev, filled, host, metro, normal_rows, padded, workspace  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# --- very negative gates ---------------------------------------------------------------

# exp2's argument is 1.443 |gate|, off by two roundings: 1.5 |gate| 2^-24 of the result, and few more behind it
DEEP_SLACK = (1.5 * 88 + 8) * 2.0 ** -24
GATES = [-16.0, -60, -64, -80, -84, -85, -86, -87, -88, -92, -96, -128, -240]
ZERO_BELOW = -126 * np.log(2)  # a sigmoid below 2^-126 counts as 0


def deep_rows(M, N, K, lift):
    """X and W of which one block of 128 columns counts: gates of row m are GATES[m], ups +-2^lift times 1 to 1.875."""
    x, w = np.zeros((M, K)), np.zeros((N, K))
    z = np.array([GATES[m % len(GATES)] for m in range(M)])
    x[:, :16] = -np.floor(-z / 16)[:, None]  # 16 times whole numbers up to 15, and 8 times the eighths of what is left
    x[:, 16:24] = (z[:, None] - 16 * x[:, :1]) / 8
    rows = np.arange(N)
    gate = rows % 16 < 8
    w[gate, :24] = 1.0
    w[~gate, 127] = (8 + rows[~gate] % 8) / 8 * np.where(rows[~gate] % 3, 1, -1)
    x[:, 127] = 1.0
    xs = np.full((M, K // 128), 127, np.uint8)
    ws = np.full((N, K // 128), 127, np.uint8)
    ws[~gate] = 127 + lift
    return x, xs, w, ws


DEEP = [(28, 544, 128, "tiled", (256, 64, 0)), (300, 288, 128, "tiled", (256, 64, 0)), (842, 13088, 640, "tiled", (256, 256, 0)),
        (14, 6272, 896, "stream", (32, 16, 1)), (45, 544, 128, "direct", None)]


@pytest.mark.parametrize("lift", [0, 40, 90])
@pytest.mark.parametrize("M,N,K,kind,plan", DEEP)
def test_swiglu_of_very_negative_gates(metro, M, N, K, kind, plan, lift):
    """Groups of 128 all of whose gates lie deep: right down to the gates whose sigmoid is 2^-126, zero below."""
    x, xs, w, ws = deep_rows(M, N, K, lift)
    codes_x, codes_w = fp8.e4m3_code(x), fp8.e4m3_code(w)
    y = fp8.values(codes_x, xs) @ fp8.values(codes_w, ws).T
    np.testing.assert_array_equal(y[:, 0], [GATES[m % len(GATES)] for m in range(M)])
    G = -(-(N // 2) // 128)
    out, scale = filled((M, G * 128)), filled((M, -(-G // 4) * 4))
    kw, X = {}, dev(codes_x)
    if kind == "direct":  # (rows of a block of 256 more than 4 GiB apart)
        kw["ldx"] = 17 << 20
        X = torch.empty((M - 1) * kw["ldx"] + K, dtype=torch.uint8, device="cuda")
        for m in range(M):
            X[m * kw["ldx"]:m * kw["ldx"] + K] = dev(codes_x[m])
    else:
        if plan[2]:
            kw["workspace"] = workspace(M, N)
        assert metro.op_gemm_fp8_plan(M, N, K, metro.EPI_FP8_SWIGLU, 0, 32 * M * N if plan[2] else 0) == (kind, *plan)
    metro.op_gemm_fp8(X, dev(padded(xs)), dev(fp8.packed_codes(codes_w)), dev(fp8.packed_bytes(ws, 0xFF)), M, N, K,
                      metro.EPI_FP8_SWIGLU, out, out_scale=scale, **kw)
    want = np.where((y[:, :1] < ZERO_BELOW), 0.0, fp8.swiglu_rows(y))
    check_rows8(host(out), host(scale)[:, :G], want, slack=DEEP_SLACK)


def test_swiglu_of_one_very_negative_row_leaves_the_others(metro):
    """A row far below does not change how the rows beside it come out."""
    M, N, K = 40, 544, 128
    x, xs, w, ws = deep_rows(M, N, K, 0)
    x[:, :127] = np.where(np.arange(M) % 2, -2 / 16, 2 / 16)[:, None]
    w, xs, ws = dev(fp8.packed_codes(fp8.e4m3_code(w))), dev(padded(xs)), dev(fp8.packed_bytes(ws, 0xFF))
    outs = []
    for deep in (False, True):
        if deep:
            x[7, :127] = -3.75
        out, scale = filled((M, 384)), filled((M, 4))
        metro.op_gemm_fp8(dev(fp8.e4m3_code(x)), xs, w, ws, M, N, K, metro.EPI_FP8_SWIGLU, out, out_scale=scale)
        outs.append((np.delete(host(out), 7, 0), np.delete(host(scale), 7, 0)))
    np.testing.assert_array_equal(outs[0][0], outs[1][0])
    np.testing.assert_array_equal(outs[0][1], outs[1][1])


# --- the norm whose sum nobody keeps ------------------------------------------------------


@pytest.mark.parametrize("rows,d", [(1, 4096), (7, 300), (40, 8192)])
def test_rmsnorm_adds_without_storing_the_sum(metro, rows, d):
    rng = np.random.default_rng(d)
    x = dev(rng.normal(size=(rows, d)).astype(np.float32))
    delta = torch.from_numpy(rng.normal(size=(rows, d)).astype(np.float32)).cuda().to(torch.bfloat16)
    g = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    before, D = x.clone(), -(-d // 128) * 128
    outs = []
    for keep in (torch.empty_like(x), None):
        h, hs = filled((rows, D)), filled((rows, -(-D // 512) * 4))
        metro.op_rmsnorm_fp8(x, g, 1e-5, h, hs, rows, d, delta=delta, x_out=keep)
        outs.append((h, hs))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and torch.equal(x, before)
    want = fp8.rms_norm(host(x).astype(np.float64) + host(delta.float()), np.ones(d), 1e-5)
    check_rows8(host(outs[1][0]), host(outs[1][1])[:, :D // 128], want)


# --- the matrix cores' sums -------------------------------------------------------------


@pytest.mark.parametrize("M,N,K,kind,ks", [(1, 32, 4736, "stream", 8), (33, 32, 2688, "tiled", 4), (69, 4224, 8960, "tiled", 8)])
def test_sums_of_normal_data_before_their_rounding(metro, M, N, K, kind, ks):
    """The k slices' fp32 sums, which stay in the workspace, against float64.  A product of two codes has 8 significant
    bits, so one within 2^5 of the largest of its eight is kept whole and a smaller one is cut by less than 2^-13 of
    the largest.  For normal data a sixth of the products is that small (|xy| < 0.07, of which the largest of eight
    is 2.2 in the mean): sqrt(1/6) * 2.2 * 2^-13 / sqrt(3) = 6.3e-5 of the result's 2-norm, at most."""
    epilogue = metro.EPI_FP8_SWIGLU if M == 69 else metro.EPI_FP8_BF16
    ws = workspace(M, N)
    assert metro.op_gemm_fp8_plan(M, N, K, epilogue, 0, 4 * ws.numel())[::3] == (kind, ks)
    rng = np.random.default_rng([M, N, K])
    x, w = normal_rows(rng, M, K), normal_rows(rng, N, K, 0.02)
    G = -(-(N // 2) // 128)
    out, scale = filled((M, G * 128 if epilogue else 2 * N)), filled((M, -(-G // 4) * 4))
    metro.op_gemm_fp8(dev(x[0]), dev(padded(x[1])), dev(fp8.packed_codes(w[0])), dev(fp8.packed_bytes(w[1], 0xFF)), M, N, K,
                      epilogue, out, out_scale=scale if epilogue else None, workspace=ws)
    got = host(ws[:ks * M * N].reshape(ks, M, N)).astype(np.float64).sum(0)
    want = fp8.values(*x) @ fp8.values(*w).T
    assert np.linalg.norm(got - want) <= 6.4e-5 * np.linalg.norm(want)
