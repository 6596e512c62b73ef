"""Which kernel makes the gradients of the matrices: the library says so itself.  No kernel is launched here."""
import ctypes

import pytest

from paper_2407_14417_amd import binding as mm
from tests.test_built_code import LIB

pytestmark = pytest.mark.skipif(not LIB.exists(), reason="needs the built library")


def small_tiles(T, d, f, E, k=1):
    rc = mm.lib().moemix_train_small_tiles(ctypes.byref(mm.CLayer(d, f, E, k, None, None, None)), T)
    assert rc >= 0, mm.lib().moe_last_error()
    return bool(rc)


# test_gpu_experts_train.py: tests that are about one of the two kernels
@pytest.mark.parametrize("counts", [(2600, 300, 9, 0, 91), (1, 2304, 1, 257, 513), (640, 576, 513, 600, 703), (3000, 1, 0, 0, 0)])
def test_large_tiles_where_the_tests_of_them_run(counts):
    assert not small_tiles(sum(counts), 1472, 2368, 5)


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 63, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("d,f", [(1088, 1984), (64, 64)])
def test_small_tiles_where_the_tests_of_them_run(rows, d, f):
    assert small_tiles(rows + 3, d, f, 16)


# (both kernels measured, backward pass in us: large and small tiles)
@pytest.mark.parametrize("T,d,f,E,small", [(64 * 32, 2048, 1408, 32, True),      # 297, 261
                                           (128 * 32, 2048, 1408, 32, True),     # 368, 346
                                           (256 * 32, 2048, 1408, 32, False),    # 542, 564
                                           (300 * 6, 320, 1408, 6, True),        # 77, 64
                                           (4096 * 2, 2048, 1408, 2, False),     # 369, 408
                                           (8 * 4, 256, 512, 4, True)])          # 33, 27
def test_the_faster_kernel_of_the_two(T, d, f, E, small):
    assert small_tiles(T, d, f, E) == small


def test_refusals():
    ask = mm.lib().moemix_train_small_tiles
    assert ask(None, 1) == mm.MOE_EINVAL and ask(ctypes.byref(mm.CLayer(100, 64, 1, 1, None, None, None)), 1) == mm.MOE_ESHAPE
