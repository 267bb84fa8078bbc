"""Products that reach each tile of csrc/wz_int8_tile.h behind each of its epilogues, and products in two launches.

Each with the tiles that it is done in, rows x columns / stages / groups of waves / bytes of K; test_product_tiles.py holds
the plan to them.  Sizes are ragged in every direction.
"""
T32, T64_32, T64 = "32x32/4/4/128", "64x32/4/2/128", "64x64/4/1/128"
T128_64, T128, T128_TWO, T128_THREE = "128x64/3/1/128", "128x128/3/1/128", "128x128/2/1/128", "128x128/3/1/64"
T192, T256 = "192x128/3/1/128", "256x256/2/1/128"
TILES = (T32, T64_32, T64, T128_64, T128, T128_TWO, T128_THREE, T192, T256)

RICH = [  # (activation, M, N, K, tiles)
    (None, 72, 303, 432, [T32]), (None, 66, 2765, 480, [T64_32]), (None, 66, 4159, 448, [T64]),
    (None, 65, 9013, 432, [T128_64]), (None, 213, 8569, 416, [T128]), (None, 402, 11511, 448, [T128_TWO]),
    (None, 140, 11001, 416, [T192]), (None, 1198, 10175, 944, [T256]), (None, 647, 10953, 464, [T128_THREE]),
    (None, 2586, 9451, 416, [T128_THREE, T64]), (None, 1044, 8165, 2032, [T128_TWO, T64]),
    (None, 1926, 8887, 1424, [T256, T64]), (None, 3461, 5251, 1632, [T256, T128]),
    ("silu", 1693, 7191, 2416, [T256]), ("silu", 2233, 7197, 944, [T128_THREE, T192]),
    ("gelu", 65, 9013, 432, [T128_64]), ("gelu", 213, 8569, 416, [T128]), ("gelu", 257, 11603, 416, [T128_TWO]),
    ("gelu", 559, 5573, 416, [T192]), ("gelu", 647, 10953, 464, [T128_THREE]), ("gelu", 2586, 9451, 416, [T128_THREE, T64])]
GATED = [
    ("silu", 72, 303, 432, [T32]), ("silu", 70, 1407, 416, [T64_32]), ("silu", 70, 2067, 432, [T64]),
    ("silu", 66, 4159, 448, [T128_64]), ("silu", 65, 9013, 432, [T128]), ("silu", 213, 8569, 416, [T128_TWO]),
    ("silu", 147, 5753, 416, [T192]), ("silu", 1674, 7683, 704, [T256]), ("silu", 257, 11603, 416, [T128_THREE]),
    ("silu", 796, 9597, 832, [T128_THREE, T192]), ("silu", 3640, 1105, 2096, [T128_TWO, T64]),
    ("silu", 815, 10455, 1424, [T256, T64]), ("silu", 845, 10315, 1808, [T256, T128]),
    ("gelu", 647, 8549, 2576, [T256]), ("gelu", 3556, 3545, 432, [T128_THREE, T64])]
