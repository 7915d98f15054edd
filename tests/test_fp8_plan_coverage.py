"""Every variant that the 8-bit products' plan chooses over a sweep of shapes is one that a GPU test runs."""

import ctypes
import math
import os
import random

import pytest


@pytest.fixture(scope="module")
def metro(repo_root):
    if not os.path.exists(os.path.join(repo_root, "paper_2411_03519_amd", "libmetro.so")):
        pytest.skip("libmetro.so not built")
    from paper_2411_03519_amd import metro
    return metro


def variant(metro, M, N, K, epilogue, E, ws):
    """What is compiled or indexed apart: kernel, tile, slices or not, epilogue, experts or not, weights past the caches."""
    shape = (M, N, K, epilogue, E, 4 * ws * M * N)
    kind, w_rows, x_rows, ks = metro.op_gemm_fp8_plan(*shape)
    return kind, w_rows, x_rows, ks > 0, epilogue, E > 0, metro.op_gemm_fp8_plan_bypass(*shape)


def test_every_variant_of_a_sweep_is_tested(metro):
    pytest.importorskip("torch")
    from tests.test_gpu_fp8_more_plans import MORE
    from tests.test_gpu_fp8_plans import VARIANTS
    tested = {variant(metro, *v[:6]) for v in VARIANTS + MORE}
    rng = random.Random(0)

    def spread(lo, hi):
        return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    seen = {}
    for _ in range(200000):
        shape = (spread(1, 16384), 32 * spread(1, 2000), 128 * spread(1, 260), rng.choice([0, 2]), rng.choice([0, 3, 8, 32, 128]),
                 rng.choice([0, 8]))
        seen.setdefault(variant(metro, *shape), shape)
    missing = {v: s for v, s in seen.items() if v not in tested}
    assert not missing, missing
    assert len(seen) >= 110


def test_plan_bypass_refusals(metro):
    def plan(M=100, N=4096, Kp=4096, epilogue=0, n_experts=0, workspace_bytes=0, out=ctypes.byref(ctypes.c_int32())):
        return metro.lib.metro_op_gemm_fp8_plan_bypass(M, N, Kp, epilogue, n_experts, workspace_bytes, out)

    assert plan() == 0
    for bad in (dict(M=0), dict(M=(1 << 26) + 1, N=32), dict(N=48), dict(Kp=200), dict(epilogue=1), dict(n_experts=-1),
                dict(n_experts=1025), dict(workspace_bytes=-1), dict(out=None)):
        assert plan(**bad) == -1 and b"gemm_fp8_plan_bypass" in metro.lib.metro_last_error(), bad
