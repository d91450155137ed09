"""Sizes of int8 projections and the way each takes with scratch, by the path that gemm_plan_i8 names: what the tests of these paths run, and what
the host's arithmetic is held to, so that other plans cannot leave a path untested."""
WAVES, FEW_WHOLE, FEW_RANGES, RANGES, TILES, SHAPES = range(6)

# (tokens, outputs, k): (path, tile rows where tiles are not chosen by the tokens alone, k ranges)
LINEAR = {
    (24, 3584, 13824): (FEW_RANGES, 0, 9), (24, 5120, 13824): (FEW_RANGES, 0, 6), (100, 5124, 13824): (FEW_RANGES, 0, 6),
    (129, 15360, 1024): (FEW_RANGES, 0, 2), (200, 5120, 13824): (FEW_RANGES, 0, 6), (256, 15360, 5120): (FEW_RANGES, 0, 2),
    (129, 15360, 512): (FEW_WHOLE, 0, 1), (201, 15364, 512): (FEW_WHOLE, 0, 1), (200, 53248, 512): (FEW_WHOLE, 0, 1),
    (810, 2564, 5120): (RANGES, 128, 3), (257, 7168, 5120): (RANGES, 160, 4), (1300, 2560, 13824): (RANGES, 192, 3),
    (1300, 12288, 8192): (TILES, 192, 3), (2000, 10240, 13824): (TILES, 256, 4), (2000, 12288, 2048): (SHAPES, 256, 1),
}
# SwiGLU: gate and up together
SWIGLU = {
    (24, 27648, 5120): (FEW_WHOLE, 0, 1), (128, 27648, 5120): (FEW_WHOLE, 0, 1), (160, 27648, 5120): (FEW_WHOLE, 0, 1),
    (256, 27648, 5120): (FEW_WHOLE, 0, 1), (200, 53248, 512): (FEW_WHOLE, 0, 1),
    (24, 3584, 13824): (FEW_RANGES, 0, 9), (65, 15360, 1024): (FEW_RANGES, 0, 2), (129, 10256, 1024): (FEW_RANGES, 0, 2), (200, 10240, 1024): (FEW_RANGES, 0, 2),
    (810, 2560, 5120): (RANGES, 128, 3), (385, 6144, 8192): (RANGES, 160, 3), (1300, 2560, 13824): (RANGES, 192, 3),
    (1300, 12288, 8192): (TILES, 192, 3), (2000, 12288, 2048): (SHAPES, 256, 1),
}
# q/k/v: (tokens, heads of queries, of keys, head_dim, hidden)
QKV = {
    (24, 64, 8, 128, 8192): (FEW_RANGES, 0, 3), (100, 64, 8, 128, 8192): (FEW_RANGES, 0, 3), (160, 104, 8, 128, 1024): (FEW_RANGES, 0, 2),
    (200, 40, 40, 128, 5120): (FEW_RANGES, 0, 2), (50, 40, 8, 64, 13824): (FEW_RANGES, 0, 9),
    (129, 104, 8, 128, 512): (FEW_WHOLE, 0, 1), (200, 352, 32, 128, 512): (FEW_WHOLE, 0, 1), (200, 208, 16, 64, 1024): (FEW_RANGES, 0, 2),
    (340, 16, 2, 128, 8192): (TILES, 128, 5), (257, 32, 4, 64, 8192): (TILES, 160, 6), (300, 64, 8, 128, 8192): (TILES, 160, 3),
    (520, 24, 8, 128, 8192): (TILES, 192, 4), (2000, 16, 2, 128, 13824): (TILES, 256, 3), (2000, 80, 8, 128, 2048): (SHAPES, 256, 1),
}


def rows():
    """(plan, "tokens features k qkv swiglu scratch") of every size."""
    for (t, n, k), plan in LINEAR.items():
        yield plan, (t, n, k, 0, 0, 1)
    for (t, n, k), plan in SWIGLU.items():
        yield plan, (t, n, k, 0, 1, 1)
    for (t, nq, nkv, d, k), plan in QKV.items():
        yield plan, (t, (nq + 2 * nkv) * d, k, 1, 0, 1)
