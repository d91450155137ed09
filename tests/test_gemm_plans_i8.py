"""Which kernel an int8 projection runs on (CPU: host arithmetic of the built library)."""
import pytest

from tests import host_program

WAVES, FEW_WHOLE, FEW_RANGES, RANGES, TILES, SHAPES = range(6)     # GemmPlanI8::Path


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = host_program.build(tmp_path_factory.mktemp("plans_i8"), "gemm_plans_i8")
    return lambda rows: host_program.run(exe, "".join("%d %d %d %d %d %d\n" % row for row in rows))


@pytest.mark.parametrize("t,n,k,swiglu", [
    # tokens, outputs, k, SwiGLU: measured slower on the waves' kernel than on the tiled ones, with weights that come from memory
    (128, 5120, 13824, 0), (65, 5120, 13824, 0), (128, 10240, 8192, 0), (65, 10240, 8192, 0), (24, 5120, 13824, 0), (64, 5120, 13824, 0),
    (24, 4096, 14336, 0), (24, 5120, 27648, 0), (24, 57344, 8192, 1), (24, 10240, 8192, 0), (64, 10240, 8192, 0), (16, 10240, 8192, 0),
    (128, 8192, 8192, 0), (128, 8192, 7168, 0), (128, 6400, 8192, 0), (16, 2048, 12800, 0),
    # short k, or few outputs, at more tokens
    (1500, 2816, 512, 1), (700, 2816, 512, 1), (1000, 2048, 512, 0), (2000, 1004, 1152, 0), (1000, 2048, 2048, 0), (520, 4096, 4096, 0),
    (200, 20480, 512, 0),
])
def test_not_on_the_waves_kernel(plans, t, n, k, swiglu):
    assert plans([(t, n, k, 0, swiglu, 1)])[0][0] != WAVES


@pytest.mark.parametrize("t,n,k,swiglu,tile", [
    # and faster there: its tile of 16, 32, 64 (two slices, one, 64 features), 128 tokens (32 features, 64)
    (1, 5120, 5120, 0, 1), (1, 15360, 5120, 0, 1), (8, 8192, 28672, 0, 1), (1, 27648, 5120, 1, 1), (16, 28672, 4096, 1, 1), (1, 25600, 5120, 1, 1),
    (1, 5120, 13824, 0, 1), (24, 15360, 5120, 0, 2), (24, 5120, 5120, 0, 2), (24, 8192, 8192, 0, 2), (64, 6144, 4096, 0, 3), (40, 5120, 5120, 0, 3),
    (64, 15360, 5120, 0, 5), (50, 12288, 4096, 0, 5), (128, 7168, 5120, 0, 6), (256, 4096, 4096, 0, 6), (128, 15360, 5120, 0, 7), (128, 11264, 5120, 1, 7),
    (256, 5120, 5120, 0, 7), (512, 4096, 4096, 0, 7), (512, 2560, 8192, 0, 7), (70, 10240, 640, 0, 4), (128, 24576, 512, 1, 4), (333, 1004, 1152, 0, 3),
    (300, 2048, 512, 0, 4),
])
def test_on_the_waves_kernel(plans, t, n, k, swiglu, tile):
    assert plans([(t, n, k, 0, swiglu, 1)])[0][:2] == (WAVES, tile)


def test_few_tokens_without_scratch_stay_there(plans):
    """Nothing else could share their k out."""
    rows = [(24, 5120, 13824), (64, 5120, 13824), (128, 5120, 13824), (24, 4096, 14336), (16, 10240, 8192), (128, 8192, 8192), (16, 2048, 12800)]
    assert all(p[0] == WAVES for p in plans([(*r, 0, 0, 0) for r in rows]))
