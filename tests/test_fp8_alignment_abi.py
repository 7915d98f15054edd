"""Every buffer of 4-byte elements is refused where it is not 4-byte aligned, on the host, before any device work (the
pointers are stand-ins and never dereferenced)."""

import pytest

from tests.test_fp8_ops_abi import BASE, GEMM, SWIGLU, lib, off, refused  # noqa: F401


def test_route_refuses_misaligned_buffers(lib):
    good = dict(logits=BASE, ldl=64, bias=BASE, T=100, n_experts=64, scoring=0, n_groups=8, top_groups=2, top_k=8,
                renormalise=1, scale=1.0, experts=BASE, weights=BASE, offsets=BASE, src=BASE, slot=BASE, workspace=BASE,
                workspace_bytes=4 * 64 * 2, stream=None)
    buffers = ("logits", "bias", "experts", "weights", "offsets", "src", "slot", "workspace")
    refused(lib, "metro_op_route", good, off(1, *buffers) + off(2, *buffers), b"misaligned")


@pytest.mark.parametrize("product", [GEMM, SWIGLU])
def test_experts_product_refuses_misaligned_indexes(lib, product):
    good = {}
    for k, v in product.items():
        if k == "W":
            good.update(x_rows=5, src=BASE, offsets=BASE, n_experts=4, R=9)
        if k != "M":
            good[k] = v
    refused(lib, "metro_op_gemm_fp8_experts", good, off(1, "src", "offsets") + off(2, "src", "offsets"), b"aligned")


def test_combine_refuses_misaligned_weights_and_slots(lib):
    good = dict(y=BASE, ldy=64, y_rows=10, weights=BASE, slot=BASE, T=5, top_k=2, d=64, resid=BASE, out=BASE, ldo=64, stream=None)
    refused(lib, "metro_op_combine_experts", good, off(2, "weights", "slot"), b"aligned")
