"""The sizes by which the product's large tiles are tested reach those tiles."""

import os

import pytest

from dense_plan import BF16, E4M3, F16, GRADIENTS, PRODUCTS, PRODUCTS_8, tile

som = pytest.importorskip("paper_2609_05138_amd.som")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(som.LIB_PATH):
        pytest.fail("libsom.so is not built (run python -m paper_2609_05138_amd.build)")
    return som.load()


def test_the_products_take_the_large_tiles(lib):
    for (M, N, K), want in PRODUCTS.items():
        for elem in (F16, BF16):
            for units in (False, True):
                for on16 in (False, True):
                    assert tile(lib, M, N, K, elem, True, units, on16) == want, (M, N, K, elem, units, on16)
        assert K // 64 > 4 and K % 64
    for (M, N, K), want in PRODUCTS_8.items():
        assert tuple(tile(lib, M, N, K, E4M3, True, True, on16) for on16 in (True, False)) == want, (M, N, K)
        assert K // 128 > 4 and K % 128
    assert set(PRODUCTS.values()) == {"256x256", "256x128", "128x128"}


def test_the_gradients_take_the_large_tiles(lib):
    for (M, N, K), (dx, dW) in GRADIENTS.items():
        for units in (False, True):
            for on16 in (False, True):
                if dx:
                    assert tile(lib, M, K, N, BF16, True, not units, on16) == dx, (M, N, K, units, on16)
                rows, cols = (N, K) if units else (K, N)
                if dW:
                    assert tile(lib, rows, cols, M, BF16, False, False, on16) == dW, (M, N, K, units, on16)
