"""How much memory the neighbour mean asks for: the sums of the segments that long rows are cut into stay in half a gigabyte (and
as much again for the last, short ones), whatever the width."""
import os

import pytest

from paper_2502_17846_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2502_17846_amd import build
        build.build_library()
    return B.load()


@pytest.mark.parametrize("d", [1, 128, 1024, 16_384, 16_385, 65_536, 262_144, 1 << 20])
@pytest.mark.parametrize("nnz", [1 << 14, 1 << 20, 1 << 26, 10 ** 10])
def test_sums_of_segments(lib, d, nnz):
    need = lib.grem_neighbour_mean_bytes(0, 1000, nnz, d, 0)
    # 2 * 2^26 sums, one row more, and 65,536 * 2 entries of the three lists beside them
    assert need <= (1 << 29) + d * 4 + (1 << 17) * 32
