"""What a layer norm's gradients ask for as scratch: room for the sums of the workgroups that the rows' way has, no more."""
import os

import pytest

from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import build as mv_build


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        mv_build.build_lib()
    return B.load()


def parts(rows, n):
    """How many pairs of rows of sums there is room for, beside the rows' two means."""
    return (B.mv_layernorm_scratch_bytes(rows, n) - 8 * rows - 16) / (8 * ((n + 3) // 4 * 4))


def test_rows_beyond_the_registers(lib):
    """At most 64 workgroups share a tile of columns, 8 where tiles are many."""
    assert parts(8192, 40_000) == 64 and parts(8192, 8193) == 64 and parts(5, 40_000) == 5
    assert parts(100_000, 1_000_000) == 8 and parts(3, 1_000_000) == 3
    assert B.mv_layernorm_scratch_bytes(8192, 40_000) < 21 << 20


def test_rows_in_registers(lib):
    """As many parts as workgroups, which is no more than rows, and at most 768, or 256 of the largest workgroups."""
    for n in (1, 64, 500, 1024, 1025, 2048, 4096, 4097, 8192):
        for rows in (1, 3, 255, 300, 2000, 100_000):
            assert 1 <= parts(rows, n) <= min(rows, 256 if n > 4096 else 768), (rows, n)
    assert parts(100_000, 2048) == 768 and parts(100_000, 8192) == 256 and parts(100_000, 4096) == 512
