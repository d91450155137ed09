"""The sizes of tests/f8b_paths.py take the paths they are there for (CPU: host arithmetic of the built library)."""
import pytest

from tests import f8b_paths, host_program


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = host_program.build(tmp_path_factory.mktemp("plans_f8b"), "gemm_plans_f8b")
    return lambda rows: host_program.run(exe, "".join("%d %d %d %d %d\n" % row for row in rows))


def test_sizes_take_their_paths(plans):
    got = plans([(*size, 1) for size in f8b_paths.SIZES])
    for (size, plan), g in zip(f8b_paths.SIZES.items(), got):
        assert g == plan, (size, g, plan)
    # every tile, whole, of each kind of output that has it: bf16, fp32 (widened codes), SwiGLU
    for kind, epilogues in (("bf16", (0, 2)), ("fp32", (1,)), ("swiglu", (3,))):
        tiles = {plan[0] for size, plan in f8b_paths.SIZES.items() if size[3] in epilogues and plan[1] == 1}
        missing = {"bf16": set(), "fp32": {f8b_paths.TILE_256}, "swiglu": {f8b_paths.ROWS_16_NARROW, f8b_paths.ROWS_32_NARROW}}[kind]
        assert tiles == set(range(9)) - missing, kind


def test_k_is_cut_only_with_scratch_and_never_through_a_block(plans):
    rows = [(t, n, k, e) for t in (1, 24, 100, 333, 1282) for n in (256, 5120) for k in (128, 1152, 13824) for e in range(4)]
    assert all(ranges == 1 for _, ranges in plans([(*r, 0) for r in rows]))
    for row, (_, ranges) in zip(rows, plans([(*r, 1) for r in rows])):
        assert 1 <= ranges <= max(1, row[2] // 256)
    # a gate matrix that ends inside a block shares a tile of partial sums with the up matrix's first rows: not cut
    assert all(ranges == 1 for _, ranges in plans([(t, 2 * 1000, 13824, 3, 1) for t in (1, 24, 100, 333, 1282)]))


def test_the_workspace_of_a_large_call_serves_smaller_ones():
    from paper_2601_11546_amd import binding as rs
    for n in (4, 512, 5120, 32000):
        sizes = [rs.relserve_linear_f8b_workspace_bytes(t, n) for t in (0, 1, 7, 64, 300, 5000, 100000)]
        assert sizes == sorted(sizes)
    for top in (0, 5, 32):
        sizes = [rs.relserve_logprobs_workspace_bytes(rows, 32000, top) for rows in (0, 1, 3, 8, 9, 200, 512, 5000)]
        assert sizes == sorted(sizes)
