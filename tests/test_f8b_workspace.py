"""The workspace of a block-scaled projection over every size that the query takes (CPU: host arithmetic of the built library)."""
import pytest

LARGEST = 2 ** 31 - 1
MOST = 64 << 20


@pytest.fixture(scope="module")
def bytes_of():
    from paper_2601_11546_amd import binding
    return binding.relserve_linear_f8b_workspace_bytes


def test_it_grows_with_either_size_up_to_64_mb(bytes_of):
    steps = [0, 1, 3, 16, 1000, 2 ** 16, 2 ** 20, 2 ** 23, 2 ** 29, 2 ** 30, LARGEST]
    got = [[bytes_of(t, n) for n in steps[1:]] for t in steps]
    for line in got + [list(column) for column in zip(*got)]:
        assert line == sorted(line)
    assert got[0][0] == 256 and max(map(max, got)) == MOST


@pytest.mark.parametrize("t,n", [(2 ** 29, 2 ** 30), (2 ** 30, 2 ** 29), (2 ** 30, 2 ** 30), (LARGEST, LARGEST), (LARGEST, 1), (1, LARGEST)])
def test_a_generous_upper_bound_serves_every_call(bytes_of, t, n):
    assert bytes_of(t, n) == MOST


def test_below_the_most_it_is_sixteen_partial_sums_of_an_output(bytes_of):
    for t, n in ((1, 5120), (24, 15360), (1023, 1024), (1024, 1023)):
        assert bytes_of(t, n) == 16 * 4 * t * n
    assert bytes_of(1024, 1024) == bytes_of(1024, 1025) == MOST
