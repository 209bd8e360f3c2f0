"""The product's plan, asked for on the host, and the sizes that the tests of its tiles use.

The library holds the plan in a C++ function that its kernels' files share; it is called
here under its linkage name."""

import ctypes

F16, BF16, E4M3 = 1, 2, 3
SHAPES = ["256x256", "256x128", "128x128", "64x128", "32x128", "16x128", "few"]

# (M, N, K): the tile that a product of it takes in 16 bits, whatever the layouts and whether
# or not rows start on 16 bytes; every one has more whole steps of k than a pipeline holds, and
# a partial one
PRODUCTS = {
    (4001, 3999, 700): "256x256",
    (3000, 3008, 1000): "256x256",
    (2500, 2500, 520): "256x128",
    (2300, 1900, 456): "256x128",
    (2048, 2048, 2000): "128x128",
    (1100, 2000, 333): "128x128",
}
# 8 bits: (rows on 16 bytes, not)
PRODUCTS_8 = {
    (4001, 3999, 700): ("256x256", "256x256"),
    (2500, 2500, 900): ("256x128", "256x128"),
    (2048, 2048, 2000): ("128x128", "128x128"),
    (3000, 3008, 1000): ("64x128", "64x128"),
}
# (M, N, K): the tiles of dx [M x K] and dW [K x N or N x K]
GRADIENTS = {
    (4001, 700, 3999): ("256x256", None),
    (700, 3999, 4001): (None, "256x256"),
    (2500, 520, 2500): ("256x128", None),
    (520, 2300, 2500): (None, "256x128"),
    (2048, 2000, 2048): ("128x128", "128x128"),
    (333, 1100, 2000): (None, "128x128"),
}


class _Plan(ctypes.Structure):
    _fields_ = [("shape", ctypes.c_int), ("splits", ctypes.c_int), ("k_split", ctypes.c_int64),
                ("partial_floats", ctypes.c_size_t)]


def tile(lib, I, J, K, elem, p_contiguous, q_contiguous, on16):
    """The tile's name of C [I][J]; `*_contiguous`: k contiguous in the operand."""
    fn = lib._ZN3som12plan_productElllibbb
    fn.restype = _Plan
    fn.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] + [ctypes.c_bool] * 3
    return SHAPES[fn(I, J, K, elem, p_contiguous, q_contiguous, on16).shape]


class _Rules(ctypes.Structure):
    _fields_ = [("few", ctypes.c_bool), ("first", ctypes.c_int), ("symmetric", ctypes.c_bool)]


class _RuledPlan(ctypes.Structure):
    _fields_ = _Plan._fields_ + [("upper", ctypes.c_bool)]


def extra(lib, I, J, K, elem, p_contiguous, q_contiguous, on16, symmetric=False):
    """(tile's name, splits of k, whether only tiles on and above the diagonal) of a product with an epilogue of
    its own."""
    fn = lib._ZN3som15plan_product_byElllibbbRKNS_9PlanRulesE
    fn.restype = _RuledPlan
    fn.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] + [ctypes.c_bool] * 3 + [ctypes.POINTER(_Rules)]
    p = fn(I, J, K, elem, p_contiguous, q_contiguous, on16, ctypes.byref(_Rules(False, 0, symmetric)))
    return SHAPES[p.shape], p.splits, p.upper


# (rows, cols) of updates whose symmetric products take 256 x 256 tiles
MIRRORED = {(4096, 4096), (4030, 4100), (4100, 4030)}


def symmetric_tile(lib, rows, cols):
    """(tile, only on and above the diagonal) of an update's A X X^T and of A A, where they are the same."""
    rows, cols = (rows + 63) // 64 * 64, (cols + 63) // 64 * 64
    tall, m = rows > cols, min(rows, cols)
    gram = extra(lib, m, m, max(rows, cols), F16, not tall, not tall, True, True)
    poly = extra(lib, m, m, m, F16, True, True, True, True)
    assert gram == poly
    return gram[0], gram[2]


# (documents, classes, features) of gradients: (splits of the scores' k axis, of dx's)
CLASSES = {
    (300, 1024, 512): (1, 1),
    (200, 600, 6000): (12, 1),
    (600, 3000, 256): (1, None),         # 6 or 8
    (8200, 16500, 24): (1, None),        # three pieces of the classes
}


def gradient_splits(lib, M, N, K, units, on16):
    n = min(N, 8192)
    return extra(lib, M, n, K, BF16, True, units, on16)[1], extra(lib, M, K, n, BF16, True, not units, on16)[1]
