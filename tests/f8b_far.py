"""Sizes of block-scaled projections whose weights are read past the caches, and of the paths that few sizes take, with the way each takes (gemm_plan_f8b: tile, k
ranges, weights past the caches): beside tests/f8b_paths.py, what the tests run and what the host's arithmetic is held to."""
from tests.f8b_paths import ROWS_16, ROWS_16_NARROW, ROWS_32, ROWS_32_NARROW, TILE_128

# (tokens, outputs, k, epilogue): (tile, k ranges, streamed)
SIZES = {
    (1, 15360, 5120, 0): (ROWS_16, 1, 1),
    (1, 15360, 5120, 1): (ROWS_16, 1, 1),
    (3, 15364, 5120, 2): (ROWS_16, 1, 1),         # outputs that end inside a tile and a block
    (16, 12288, 4096, 1): (ROWS_16, 1, 1),
    (16, 27648, 5120, 3): (ROWS_16, 1, 1),
    (1, 17308, 3968, 2): (ROWS_16, 2, 1),
    (2, 1392, 24192, 1): (ROWS_16, 3, 1),
    (1, 1280, 26496, 3): (ROWS_16, 6, 1),
    (7, 20000, 1664, 1): (ROWS_16, 1, 0),         # just below 32 MB
    (5, 48, 22144, 0): (ROWS_16_NARROW, 16, 0),
    (1, 512, 14336, 0): (ROWS_16_NARROW, 16, 0),
    (18, 4, 72448, 0): (ROWS_32_NARROW, 16, 0),
    (67, 1444, 21760, 1): (ROWS_32, 3, 0),
    (33765, 4, 1152, 0): (TILE_128, 3, 0),
}
