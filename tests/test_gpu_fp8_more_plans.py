"""The variants of the 8-bit products that test_gpu_fp8_plans.py does not name: weights past the caches (kernels of their
own), and k slices of the largest tiles.  Whole numbers, so that results have to be exact, as there."""

import pytest

from tests.test_gpu_fp8_plans import metro, run  # noqa: F401

pytestmark = pytest.mark.gpu

# (rows, N, K, epilogue, experts (0: dense), workspace in slices, kind, W rows, X rows, k slices, weights past the caches)
MORE = [
    (6, 19744, 4864, 0, 0, 8, "tiled", 128, 64, 0, True),
    (7, 6592, 4864, 0, 3, 8, "tiled", 128, 64, 0, True),
    (2, 3616, 26624, 0, 0, 8, "tiled", 128, 64, 8, True),
    (7, 1216, 26368, 0, 3, 8, "tiled", 128, 64, 8, True),
    (4, 1056, 30464, 2, 3, 8, "tiled", 128, 64, 8, True),
    (119, 25056, 3840, 0, 0, 0, "tiled", 128, 128, 0, True),
    (175, 7616, 4224, 0, 3, 0, "tiled", 128, 128, 0, True),
    (189, 2240, 14336, 0, 3, 8, "tiled", 128, 128, 4, True),
    (68, 7776, 12416, 2, 0, 8, "tiled", 128, 128, 4, True),
    (178, 5120, 6272, 2, 3, 8, "tiled", 128, 128, 2, True),
    (132, 30336, 3200, 0, 0, 8, "tiled", 128, 192, 0, True),
    (376, 8416, 3840, 0, 3, 8, "tiled", 128, 192, 0, True),
    (130, 3168, 30848, 0, 0, 8, "tiled", 128, 192, 8, True),
    (238, 2432, 13184, 0, 3, 8, "tiled", 128, 192, 4, True),
    (169, 7168, 13440, 2, 0, 8, "tiled", 128, 192, 4, True),
    (366, 4480, 7296, 2, 3, 8, "tiled", 128, 192, 2, True),
    (197, 20352, 4736, 0, 0, 0, "tiled", 128, 256, 0, True),
    (366, 10016, 3200, 0, 3, 8, "tiled", 128, 256, 0, True),
    (211, 5856, 16640, 0, 0, 8, "tiled", 128, 256, 4, True),
    (876, 2784, 11520, 0, 3, 8, "tiled", 128, 256, 2, True),
    (209, 10624, 9088, 2, 0, 8, "tiled", 128, 256, 2, True),
    (355, 2400, 13568, 2, 3, 8, "tiled", 128, 256, 4, True),
    (1, 46880, 2048, 0, 0, 0, "tiled", 256, 64, 0, True),
    (4, 14720, 2176, 2, 3, 8, "tiled", 256, 64, 0, True),
    (1, 5344, 18048, 0, 0, 8, "tiled", 256, 64, 8, True),
    (5, 1504, 21632, 0, 3, 8, "tiled", 256, 64, 8, True),
    (3, 5216, 18432, 2, 0, 8, "tiled", 256, 64, 8, True),
    (6, 2176, 14720, 2, 3, 8, "tiled", 256, 64, 8, True),
    (92, 37568, 2560, 0, 0, 8, "tiled", 256, 128, 0, True),
    (135, 22784, 1408, 0, 3, 0, "tiled", 256, 128, 0, True),
    (72, 34112, 2816, 2, 0, 0, "tiled", 256, 128, 0, True),
    (237, 13184, 2432, 2, 3, 0, "tiled", 256, 128, 0, True),
    (99, 4864, 19840, 0, 0, 8, "tiled", 256, 128, 8, True),
    (182, 1696, 19200, 0, 3, 8, "tiled", 256, 128, 8, True),
    (91, 4512, 21504, 2, 0, 8, "tiled", 256, 128, 8, True),
    (216, 3328, 9728, 2, 3, 8, "tiled", 256, 128, 4, True),
    (168, 46880, 2048, 0, 0, 8, "tiled", 256, 192, 0, True),
    (263, 22848, 1408, 0, 3, 0, "tiled", 256, 192, 0, True),
    (354, 15744, 2048, 2, 3, 8, "tiled", 256, 192, 0, True),
    (2353, 800, 9728, 0, 0, 8, "tiled", 256, 192, 4, False),
    (131, 9376, 12160, 0, 0, 8, "tiled", 256, 192, 4, True),
    (2614, 704, 9216, 0, 3, 8, "tiled", 256, 192, 4, False),
    (670, 2688, 12288, 0, 3, 8, "tiled", 256, 192, 4, True),
    (806, 2336, 9216, 2, 0, 8, "tiled", 256, 192, 4, False),
    (136, 4992, 20480, 2, 0, 8, "tiled", 256, 192, 8, True),
    (3439, 1056, 6400, 2, 3, 8, "tiled", 256, 192, 2, False),
    (877, 4544, 7424, 2, 3, 8, "tiled", 256, 192, 2, True),
    (453, 24352, 3968, 0, 0, 8, "tiled", 256, 256, 0, True),
    (451, 17312, 1920, 0, 3, 0, "tiled", 256, 256, 0, True),
    (211, 41792, 2304, 2, 0, 0, "tiled", 256, 256, 0, True),
    (379, 19232, 1664, 2, 3, 8, "tiled", 256, 256, 0, True),
    (1407, 2080, 15616, 0, 0, 8, "tiled", 256, 256, 4, False),
    (194, 4384, 22400, 0, 0, 8, "tiled", 256, 256, 8, True),
    (1767, 1440, 13184, 0, 3, 8, "tiled", 256, 256, 4, False),
    (866, 2688, 13312, 0, 3, 8, "tiled", 256, 256, 4, True),
    (1754, 1664, 14720, 2, 0, 8, "tiled", 256, 256, 4, False),
    (197, 8672, 11136, 2, 0, 8, "tiled", 256, 256, 4, True),
    (4635, 544, 12800, 2, 3, 8, "tiled", 256, 256, 4, False),
    (870, 2624, 13824, 2, 3, 8, "tiled", 256, 256, 4, True),
]


@pytest.mark.parametrize("M,N,K,epilogue,E,ws,kind,w_rows,x_rows,ks,bypass", MORE)
def test_variant(metro, M, N, K, epilogue, E, ws, kind, w_rows, x_rows, ks, bypass):
    shape = (M, N, K, epilogue, E, 4 * ws * M * N)
    assert metro.op_gemm_fp8_plan(*shape) == (kind, w_rows, x_rows, ks)
    assert metro.op_gemm_fp8_plan_bypass(*shape) == bypass
    run(metro, M, N, K, epilogue, E, ws)
