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


# rows off 16 bytes, k contiguous in both: the best of all tiles by measured times (us: this one,
# and the one that a step through registers priced at twice and more of its time led to)
RAGGED = {
    (2001, 1001, 2003): "64x128",     # 24.3; 128x128 in two splits 29.4
    (129, 4097, 1025): "64x128",      # 13.0 (32x128 12.4); 128x128 in three splits 16.5
    (333, 1023, 5001): "64x128",      # 20.2; 128x128 in eight splits 21.9
    (200, 1000, 10001): "64x128",     # 20.1; 128x128 in sixteen splits 22.1
    (4001, 3999, 4001): "256x256",
}


def test_rows_off_16_bytes_take_the_best_tiles(lib):
    for (M, N, K), want in RAGGED.items():
        assert tile(lib, M, N, K, BF16, True, True, False) == want, (M, N, K)
