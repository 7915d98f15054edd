"""Refusals of the 8-bit feed-forward operators: found on the host before any device work, so they run without a GPU (the
pointers are stand-ins and never dereferenced)."""

import ctypes
import os

import pytest

P = ctypes.c_void_p
BASE = 1 << 20  # a stand-in device address, 16-byte aligned


@pytest.fixture(scope="module")
def lib(repo_root):
    if not os.path.exists(os.path.join(repo_root, "paper_2411_03519_amd", "libmetro.so")):
        pytest.skip("libmetro.so not built")
    from paper_2411_03519_amd import metro
    return metro.lib


def refused(lib, name, good, changes, word=b""):
    """Every change of one argument of the good call is refused with E_INVAL and a message."""
    fn = getattr(lib, name)
    keys = list(good)
    for change in changes:
        args = {**good, **change}
        assert fn(*[P(args[k]) if k in POINTERS else args[k] for k in keys]) == -1, (name, change)
        msg = lib.metro_last_error()
        assert msg and word in msg, (name, change, msg)


POINTERS = {"W_rowmajor", "W_packed", "W_scale", "x", "delta", "g", "x_out", "h_bf16", "h", "h_scale", "X", "x_scale", "W",
            "w_scale", "out_bf16", "out_fp8", "out_scale", "workspace", "stream", "logits", "bias", "experts", "weights",
            "offsets", "src", "slot", "y", "resid", "out"}


def nulls(*names):
    return [{n: None} for n in names]


def off(by, *names):
    return [{n: BASE + by} for n in names]


def test_pack_weight_refusals(lib):
    good = dict(W_rowmajor=BASE, ld=256, N=32, K=256, Kp=256, W_packed=BASE, W_scale=BASE, stream=None)
    refused(lib, "metro_op_pack_weight_fp8", good, nulls("W_rowmajor", "W_packed", "W_scale") + off(8, "W_packed", "W_scale") +
            [{"N": 24}, {"N": 0}, {"N": -16}, {"K": 0}, {"K": 257}, {"Kp": 320}, {"Kp": 0}, {"ld": 255}])


def test_rmsnorm_refusals(lib):
    good = dict(x=BASE, ldx=256, delta=BASE, ldd=256, g=BASE, eps=1e-5, x_out=BASE, h_bf16=BASE, ldh_bf16=256, h=BASE, ldh=256,
                h_scale=BASE, lds=4, rows=3, d=256, stream=None)
    refused(lib, "metro_op_rmsnorm_fp8", good, nulls("x", "g", "h", "h_scale", "delta") + off(8, "x", "x_out") +
            off(4, "delta", "g", "h_bf16") + off(2, "h") +
            [{"rows": -1}, {"d": 0}, {"d": 254}, {"d": 8196, "ldx": 9000, "ldd": 9000, "ldh": 9000, "ldh_bf16": 9000, "lds": 80},
             {"ldx": 252}, {"ldx": 258}, {"ldd": 252}, {"ldd": 257}, {"ldh_bf16": 252}, {"ldh_bf16": 258}, {"ldh": 252},
             {"ldh": 258}, {"lds": 1}, {"d": 132, "ldh": 132}])


GEMM = dict(X=BASE, ldx=512, x_scale=BASE, ldxs=4, W=BASE, w_scale=BASE, Kp=512, M=5, N=320, epilogue=0, out_bf16=BASE,
            out_fp8=None, ldo=320, out_scale=None, ldos=0, workspace=None, workspace_bytes=0, stream=None)
SWIGLU = dict(GEMM, epilogue=2, out_bf16=None, out_fp8=BASE, ldo=256, out_scale=BASE, ldos=2)
OPERANDS = (nulls("X", "x_scale", "W", "w_scale") + off(8, "X", "W", "w_scale", "workspace") + off(2, "x_scale") +
            [{"ldx": 500}, {"ldx": 520}, {"ldxs": 3}, {"ldxs": 6}, {"Kp": 500}, {"Kp": 0}, {"N": 336}, {"N": 0}, {"N": -32},
             {"Kp": 640, "ldx": 640}, {"epilogue": 1}, {"epilogue": 3}, {"workspace_bytes": -1}])


def test_gemm_refusals(lib):
    refused(lib, "metro_op_gemm_fp8", GEMM, OPERANDS + nulls("out_bf16") + off(4, "out_bf16") +
            [{"M": -1}, {"M": (1 << 26) + 1}, {"M": 1 << 26, "N": 1056, "ldo": 1056}, {"ldo": 316}, {"ldo": 322}], b"gemm_fp8")
    refused(lib, "metro_op_gemm_fp8", SWIGLU, OPERANDS + nulls("out_fp8", "out_scale") + off(8, "out_fp8") +
            [{"M": -1}, {"ldo": 160}, {"ldo": 264}, {"ldos": 1}], b"gemm_fp8")


def test_experts_refusals(lib):
    def by_experts(g):
        d = {}
        for k, v in g.items():
            if k == "W":
                d.update(x_rows=5, src=BASE, offsets=BASE, n_experts=4, R=9)
            if k != "M":
                d[k] = v
        return d

    more = nulls("offsets") + [{"n_experts": 0}, {"n_experts": 1025}, {"R": -1}, {"x_rows": 0}, {"x_rows": -1}, {"src": None}]
    refused(lib, "metro_op_gemm_fp8_experts", by_experts(GEMM), OPERANDS + more + nulls("out_bf16"), b"gemm_fp8_experts")
    refused(lib, "metro_op_gemm_fp8_experts", by_experts(SWIGLU), OPERANDS + more + nulls("out_fp8", "out_scale"),
            b"gemm_fp8_experts")


def test_route_refusals(lib):
    good = dict(logits=BASE, ldl=64, bias=None, T=100, n_experts=64, scoring=0, n_groups=8, top_groups=2, top_k=8,
                renormalise=1, scale=1.0, experts=BASE, weights=BASE, offsets=BASE, src=BASE, slot=BASE, workspace=BASE,
                workspace_bytes=4 * 64 * 2, stream=None)
    refused(lib, "metro_op_route", good, nulls("logits", "experts", "weights", "offsets", "src", "slot", "workspace") +
            [{"T": -1}, {"ldl": 63}, {"n_experts": 0}, {"n_experts": 513, "ldl": 513}, {"scoring": 2}, {"n_groups": 0},
             {"n_groups": 7}, {"n_groups": 128}, {"top_groups": 0}, {"top_groups": 9}, {"top_k": 0}, {"top_k": 17}, {"top_k": 33},
             {"workspace_bytes": 4 * 64 * 2 - 1}, {"T": (1 << 24) + 1, "workspace_bytes": 1 << 40}], b"route")


def test_combine_refusals(lib):
    good = dict(y=BASE, ldy=64, y_rows=10, weights=BASE, slot=BASE, T=5, top_k=2, d=64, resid=BASE, out=BASE, ldo=64, stream=None)
    refused(lib, "metro_op_combine_experts", good, nulls("y", "weights", "slot", "out") + off(8, "y", "resid", "out") +
            [{"T": -1}, {"y_rows": -1}, {"top_k": 0}, {"d": 0}, {"d": 60}, {"ldy": 56}, {"ldy": 68}, {"ldo": 60}, {"ldo": 66}])


def test_plan_refusals(lib):
    v = [ctypes.c_int32() for _ in range(4)]

    def plan(M=100, N=4096, Kp=4096, epilogue=0, n_experts=0, workspace_bytes=0, out=v):
        return lib.metro_op_gemm_fp8_plan(M, N, Kp, epilogue, n_experts, workspace_bytes, *[None if x is None else ctypes.byref(x) for x in out])

    assert plan() == 0 and plan(M=1 << 24) == 0
    for bad in (dict(M=0), dict(M=(1 << 26) + 1, N=32), dict(M=(1 << 24) + 1), dict(N=48), dict(Kp=200), dict(epilogue=1),
                dict(n_experts=-1), dict(n_experts=1025), dict(workspace_bytes=-1), dict(out=v[:3] + [None])):
        assert plan(**bad) == -1 and b"gemm_fp8_plan" in lib.metro_last_error(), bad


def test_calls_without_rows_take_empty_buffers(lib):
    """Tensors without elements have address 0; nothing is launched for them."""
    norm = [P(None), 256, P(None), 256, P(BASE), 1e-5, P(None), P(None), 256, P(None), 256, P(None), 4, 0, 256, P(None)]
    assert lib.metro_op_rmsnorm_fp8(*norm) == 0
    for epilogue, ldo, ldos in ((0, 320, 0), (2, 256, 2)):
        tail = [512, 0, 320, epilogue, P(None), P(None), ldo, P(None), ldos, P(None), 0, P(None)]
        assert lib.metro_op_gemm_fp8(P(None), 512, P(None), 4, P(BASE), P(BASE), *tail) == 0
        tail[1:3] = [320]
        assert lib.metro_op_gemm_fp8_experts(P(None), 512, P(None), 4, 0, P(None), P(BASE), 4, 0, P(BASE), P(BASE), *tail) == 0
    assert lib.metro_op_combine_experts(P(None), 64, 0, P(None), P(None), 0, 2, 64, P(None), P(None), 64, P(None)) == 0


def test_widths_past_2_to_30_are_refused(lib):
    for change in ({"M": 1, "N": (1 << 30) + 32, "ldo": (1 << 30) + 32}, {"M": 1, "N": (1 << 31) - 32, "ldo": (1 << 31) - 4}):
        refused(lib, "metro_op_gemm_fp8", GEMM, [change], b"2^30")
    v = [ctypes.c_int32() for _ in range(4)]
    assert lib.metro_op_gemm_fp8_plan(1, (1 << 31) - 32, 128, 0, 0, 0, *[ctypes.byref(x) for x in v]) == -1
    assert lib.metro_op_gemm_fp8_plan(1, 1 << 30, 128, 0, 0, 0, *[ctypes.byref(x) for x in v]) == 0
