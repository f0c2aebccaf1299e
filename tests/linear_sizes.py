"""Sizes of switch_linear (bf16) whose products take the 256 x 256 tiles: test_operators_launches.py holds the
library to that choice, test_linear_tiles_gpu.py runs them.  No dimension is a multiple of the tile, no k of its step."""

# M, K, N, activation, dropout, k in parts
LARGE_FORWARD = [
    (5965, 232, 2224, "none", 0.1, False), (4265, 4208, 992, "relu", 0.0, True), (2455, 248, 4944, "relu", 0.1, False),
    (2438, 1400, 5416, "gelu", 0.0, False), (1053, 4944, 3752, "gelu", 0.1, True), (3744, 728, 2120, "geglu", 0.1, False),
    (2057, 5184, 984, "geglu", 0.0, True),
]
# M, K, N, activation, dropout, columns of dx in parts, rows of dW in parts
LARGE_BACKWARD = [
    (6564, 1488, 496, "none", 0.1, False, True), (1167, 5960, 792, "none", 0.0, False, False),
    (6186, 1000, 648, "relu", 0.1, False, True), (979, 5920, 1056, "relu", 0.0, False, False),
    (2823, 2984, 728, "gelu", 0.1, False, True), (1410, 4816, 1144, "gelu", 0.0, False, False),
    (385, 4152, 4584, "gelu", 0.1, True, False), (8929, 744, 512, "geglu", 0.1, False, True),
    (1559, 5312, 416, "geglu", 0.0, False, False), (390, 1952, 4728, "geglu", 0.25, True, False),
]
