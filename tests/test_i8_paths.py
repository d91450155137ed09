"""The sizes of tests/i8_paths.py take the paths they are there for (CPU: host arithmetic of the built library)."""
from tests import host_program, i8_paths


def test_sizes_take_their_paths(tmp_path):
    sizes = list(i8_paths.rows())
    got = host_program.run(host_program.build(tmp_path, "gemm_plans_i8"), "".join("%d %d %d %d %d %d\n" % row for _, row in sizes))
    for (plan, row), g in zip(sizes, got):
        assert g[:3] == plan, (row, g, plan)
        assert (g[3] > 0) == (plan[0] == i8_paths.TILES) and (g[4] > 0) == (plan[0] == i8_paths.SHAPES)
    assert {plan[0] for plan, _ in sizes} == {i8_paths.FEW_WHOLE, i8_paths.FEW_RANGES, i8_paths.RANGES, i8_paths.TILES, i8_paths.SHAPES}
