"""Shapes of products for every way in which one is cut (csrc/tahq_mx4_plan.hpp): no edge is a multiple of a tile's, and groups of 256 columns
leave every remainder of the buffers' rounds; 70, 300, 1100, 1300 and 2100 end in a stage of 128 columns that is not there."""

# kind: -1 few rows of A, then the tiles of kTiles; parts: whether the sum over k is cut into runs
FEW, T256, T256x128, T128, T64x128, T64, T64_TEAMS = range(-1, 6)

# (kind, parts, type of C, m, n, k)
PRODUCTS = [
    (FEW, False, "bf16", 1, 1601, 1600), (FEW, False, "f32", 16, 333, 2047), (FEW, False, "bf16", 31, 515, 1100), (FEW, False, "f32", 17, 99, 70),
    (T256, False, "bf16", 3716, 3237, 1300), (T256, False, "bf16", 2984, 2703, 1700), (T256, False, "bf16", 3411, 2347, 2100),
    (T256, False, "f32", 3777, 3237, 2300), (T256, False, "f32", 2984, 2703, 3300),
    (T256x128, False, "bf16", 3716, 2703, 70), (T256x128, False, "bf16", 3716, 2703, 300), (T256x128, False, "bf16", 3716, 3237, 600),
    (T256x128, False, "bf16", 2557, 1635, 2700), (T256x128, False, "bf16", 1154, 3415, 3000), (T256x128, False, "bf16", 1154, 3415, 3300),
    (T256x128, False, "f32", 3350, 3593, 70), (T256x128, False, "f32", 3350, 3593, 300), (T256x128, False, "f32", 3350, 3593, 600),
    (T256x128, False, "f32", 3350, 3593, 1100),
    (T128, False, "bf16", 2313, 835, 70), (T128, False, "bf16", 2313, 835, 300), (T128, False, "bf16", 2313, 835, 600),
    (T128, False, "f32", 3777, 1546, 300), (T128, False, "f32", 2313, 835, 600), (T128, False, "f32", 2313, 835, 1100),
    (T64x128, False, "bf16", 202, 4127, 300), (T64x128, False, "bf16", 202, 4127, 1100), (T64x128, False, "f32", 202, 4127, 600),
    (T64, False, "bf16", 33, 51, 600), (T64, False, "bf16", 77, 51, 900), (T64, False, "f32", 33, 51, 1100),
    (T64_TEAMS, False, "bf16", 33, 51, 3300), (T64_TEAMS, False, "f32", 99, 130, 3000),
    (T64, True, "bf16", 41, 67, 16384), (T64, True, "f32", 201, 131, 20000), (T64, True, "f32", 70, 66, 12500),
]
