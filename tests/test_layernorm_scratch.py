"""What a layer norm's gradients ask for as scratch: room for the sums of the workgroups that the rows' way has, and not less than
smaller calls ask for."""
import os

import pytest

from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import build as mv_build


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        mv_build.build_lib()
    return B.load()


def sums(rows, n):
    """Bytes beside the rows' two means."""
    return B.mv_layernorm_scratch_bytes(rows, n) - 8 * rows - 16


def parts(count, n):
    """Of so many pairs of rows of sums."""
    return count * 8 * ((n + 3) // 4 * 4)


def test_rows_beyond_the_registers(lib):
    """At most 64 workgroups share a tile of columns, 8 where tiles are many; shorter rows, of which 512 workgroups each have 4096
    sums of both kinds, 16.8 MB."""
    assert sums(8192, 40_000) == parts(64, 40_000) and sums(8192, 8193) == parts(512, 4096) and sums(5, 40_000) == parts(5, 40_000)
    assert sums(100_000, 10_000_000) == parts(8, 10_000_000) and sums(3, 1_000_000) == parts(3, 1_000_000)
    assert B.mv_layernorm_scratch_bytes(8192, 40_000) < 21 << 20


def test_rows_in_registers(lib):
    """As many parts as workgroups, which is no more than rows, and at most 768, or 256 of the largest workgroups."""
    for n in (1, 64, 500, 1024, 1025, 2048, 4096, 4097, 8192):
        for rows in (1, 3, 255, 300, 2000, 100_000):
            assert parts(1, n) <= sums(rows, n) <= max(parts(min(rows, 256 if n > 4096 else 768), n), parts(min(rows, 512), 4096)), (rows, n)
    assert sums(100_000, 2048) == parts(768, 2048) and sums(100_000, 8192) == parts(256, 8192) and sums(100_000, 4096) == parts(512, 4096)


def test_the_largest_call_is_enough_for_all(lib):
    """A program keeps scratch for its largest call and gives it to the others."""
    sizes = sorted({v for e in range(22) for v in (2 ** e - 1, 2 ** e, 2 ** e + 1, 5 * 2 ** e) if v > 0} | {129_023, 129_024, 129_025, 131_071})
    for rows in (1, 3, 100, 255, 256, 257, 700, 1024, 1537, 50_000):
        need = [B.mv_layernorm_scratch_bytes(rows, n) for n in sizes]
        assert need == sorted(need), rows
    for n in sizes:
        need = [B.mv_layernorm_scratch_bytes(rows, n) for rows in sizes]
        assert need == sorted(need), n
