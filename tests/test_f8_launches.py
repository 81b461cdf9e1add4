"""Which kernel a product with an 8-bit weight takes (host arithmetic, no GPU): the launches that the GPU tests rely on."""
import ctypes as C

import pytest

import paper_2312_04916_amd as ee
from test_gpu_f8 import SIZES
from test_gpu_f8_forms import FEW, TILES


def test_arguments_are_checked():
    s, L = (C.c_int32 * 4)(), ee.lib()
    for args, code in (((1, 1, 1, 0), 0), ((1 << 20, 1 << 22, 1 << 18, 1), 0), ((0, 1, 1, 0), -7), (((1 << 20) + 1, 1, 1, 0), -7), ((1, 0, 1, 0), -1), ((1, 1, (1 << 18) + 1, 0), -1)):
        assert L.ee_debug_f8_launch(*args, s) == code, args
    assert L.ee_debug_f8_launch(1, 1, 1, 0, None) == -7


@pytest.mark.parametrize("m,n,k,pair,launch", FEW)
def test_few_rows(m, n, k, pair, launch):
    assert ee.f8_launch(m, n, k, pair) == launch


@pytest.mark.parametrize("m,n,k,pair,tile", TILES)
def test_tiles_through_lds(m, n, k, pair, tile):
    assert ee.f8_launch(m, n, k, pair) == (*tile, 4, 2)


def test_the_tests_reach_every_launch():
    """All kinds of the rule: six tiles, each for single weights and pairs; twelve of rows that go into registers."""
    reached = {ee.f8_launch(m, n, k, pair) + (pair,) for m, n, k, pair, _ in TILES}
    assert len(reached) == 12 and {r[:2] for r in reached} == {(256, 256), (256, 192), (192, 192), (256, 128), (128, 192), (128, 128)}
    streams = {ee.f8_launch(m, n, k, pair) for m, n, k in SIZES for pair in (False, True)} | {ee.f8_launch(*f[:4]) for f in FEW}
    assert streams == {(16, 16, 8, 1), (16, 32, 8, 1), (16, 16, 4, 0), (16, 32, 4, 0), (16, 32, 8, 0), (32, 16, 4, 0), (32, 16, 8, 0), (32, 32, 4, 0), (64, 16, 4, 0),
                       (64, 32, 4, 0), (64, 64, 4, 0), (128, 64, 4, 0)}


def test_workspace_goes_with_the_launch():
    b = C.c_size_t()
    for m, k in ((1, 1), (1, 32768), (1, 32769), (16, 2048), (16, 2049), (17, 1), (100, 500)):
        assert ee.lib().ee_f8_matmul_bytes(m, 300, k, 0, ee.EE_BF16, C.byref(b)) == 0
        assert (b.value == 0) == (ee.f8_launch(m, 300, k)[3] == 1), (m, k)
