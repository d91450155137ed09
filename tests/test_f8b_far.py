"""The sizes of tests/f8b_far.py take the paths they are there for (CPU: host arithmetic of the built library)."""
import pytest

from tests import f8b_far, f8b_paths, host_program


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = host_program.build(tmp_path_factory.mktemp("streams_f8b"), "gemm_streams_f8b")
    return lambda rows: host_program.run(exe, "".join("%d %d %d %d 1\n" % row for row in rows))


def test_sizes_take_their_paths(plans):
    for (size, plan), got in zip(f8b_far.SIZES.items(), plans(f8b_far.SIZES)):
        assert got == plan, (size, got, plan)
    # weights past the caches: whole for every kind of output, in k ranges on codes and on widened codes
    streamed = {(size[3], plan[1] > 1) for size, plan in f8b_far.SIZES.items() if plan[2]}
    assert {(e, False) for e in range(4)} <= streamed and (1, True) in streamed and ({(0, True), (2, True), (3, True)} & streamed)


def test_every_tile_that_k_ranges_can_take_is_tested(plans):
    """Partial sums have one kernel for each tile, on codes and on widened codes."""
    both = [(size, plan[:2]) for size, plan in {**f8b_paths.SIZES, **f8b_far.SIZES}.items()]
    tested = {(size[3] == 1, plan[0]) for size, plan in both if plan[1] > 1}
    rows = [(t, n, k, e) for t in (1, 5, 18, 40, 70, 100, 128, 200, 400, 700, 1300, 3000, 8000, 34000)
            for n in (4, 36, 256, 1024, 1444, 2560, 5120, 17308) for k in (1152, 2688, 5120, 13824, 21760, 72448) for e in range(4)
            if t * k < 2 ** 31 and n * k < 2 ** 31 and (e < 3 or n % 16 == 0)]
    taken = {(row[3] == 1, tile) for row, (tile, ranges, _) in zip(rows, plans(rows)) if ranges > 1}
    assert taken <= tested, taken - tested
    assert {tile for wide, tile in tested if not wide} == set(range(9))


def test_only_few_tokens_stream_large_weights(plans):
    rows = [(t, n, 5120, e) for t in (1, 16, 17, 24, 64, 300, 2000) for n in (4096, 6544, 6560, 15360, 27648) for e in range(4)]
    for row, (tile, _, streamed) in zip(rows, plans(rows)):
        assert streamed == (tile == f8b_paths.ROWS_16 and row[1] * row[2] >= 32 << 20), row
        assert not streamed or row[0] <= 16
