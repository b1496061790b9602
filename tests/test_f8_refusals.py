"""Arguments that the 8-bit calls refuse, all before any device call: the addresses here are made up."""
import os

import pytest

from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import build as mv_build

P = 1 << 20            # an address with every alignment


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        mv_build.build_lib()
    return B.load()


def test_sizes(lib):
    assert [B.mv_f8_row_bytes(n) for n in (0, 1, 128, 129, 500, (1 << 31) - 1, 1 << 31)] == [0, 128, 128, 256, 512, 1 << 31, 0]
    assert [B.mv_f8_row_scales(n) for n in (0, 1, 128, 512, 513, (1 << 31) - 1, -5)] == [0, 4, 4, 4, 8, 1 << 24, 0]
    for f in (B.mv_f8_product_scratch_bytes, B.mv_f8_linear_scratch_bytes, B.mv_f8_linear_grad_scratch_bytes):
        assert f(0, 1, 1) == 0 and f(1, 1 << 31, 1) == 0 and f(1, 1, -1) == 0
    assert B.mv_f8_linear_grad_scratch_bytes(100, 100, 100) > 0


# every call with good arguments by name, in the order of the C declaration
CALLS = {
    "mv_f8_encode": dict(vals=P, dtype=0, ld_vals=300, rows=4, n=300, codes=2 * P, ld_bytes=384, scales=3 * P, ld_scales=4, stream=None),
    "mv_f8_encode_t": dict(vals=P, dtype=0, ld_vals=300, rows=4, n=300, codes=2 * P, ld_bytes=128, scales=3 * P, ld_scales=4, stream=None),
    "mv_f8_decode": dict(codes=2 * P, ld_bytes=384, scales=3 * P, ld_scales=4, rows=4, n=300, out=P, dtype=0, ld_out=300, stream=None),
    "mv_f8_product": dict(a_codes=P, ld_ab=384, a_scales=2 * P, ld_as=4, b_codes=3 * P, ld_bb=384, b_scales=4 * P, ld_bs=4, m=4, n=300,
                          k=300, c=5 * P, c_dtype=0, ld_c=300, scratch=6 * P, scratch_bytes=1 << 20, stream=None),
    "mv_f8_linear": dict(x=P, x_dtype=0, ld_x=300, w_codes=3 * P, ld_bytes=384, w_scales=4 * P, ld_scales=4, m=40, n=300, k=300, y=5 * P,
                         y_dtype=0, ld_y=300, scratch=6 * P, scratch_bytes=1 << 20, stream=None),
    "mv_f8_linear_grad": dict(x=P, ld_x=300, dy=2 * P, ld_dy=300, dtype=0, wt_codes=3 * P, ld_bytes=384, wt_scales=4 * P, ld_scales=4,
                              m=40, n=300, k=300, dx=5 * P, dx_dtype=0, ld_dx=300, dw=7 * P, dw_dtype=0, ld_dw=300, scratch=6 * P,
                              scratch_bytes=1 << 24, stream=None),
}
POINTERS = {"vals": 2, "codes": 8, "scales": 2, "out": 2, "a_codes": 8, "a_scales": 2, "b_codes": 8, "b_scales": 2, "c": 2,
            "x": 2, "w_codes": 8, "w_scales": 2, "y": 2, "dy": 2, "wt_codes": 8, "wt_scales": 2}
OPTIONAL = {"dx": 2, "dw": 2}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_arguments(lib, name):
    good, call = CALLS[name], getattr(lib, name)

    def status(**change):
        return call(*{**good, **change}.values())

    bad = [{p: 0} for p in POINTERS if p in good]
    bad += [{p: good[p] + off} for p, off in {**POINTERS, **OPTIONAL}.items() if p in good]
    for size in ("rows", "m", "n", "k"):
        if size in good:
            bad += [{size: 0}, {size: -1}, {size: 1 << 31}]
    for ld in good:
        if ld.startswith("ld_"):
            bad += [{ld: 0}, {ld: good[ld] - 1}]
            if ld in ("ld_bytes", "ld_ab", "ld_bb"):
                bad += [{ld: good[ld] + 8}]
            if ld in ("ld_scales", "ld_as", "ld_bs"):
                bad += [{ld: good[ld] + 2}]
        if ld.endswith("dtype"):
            bad += [{ld: 2}, {ld: -1}]
    if name in ("mv_f8_linear", "mv_f8_linear_grad"):
        bad += [{"scratch": 0}, {"scratch": good["scratch"] + 8}, {"scratch_bytes": 64}]
    if name == "mv_f8_linear_grad":
        bad += [{"dx": 0, "dw": 0}]
    for change in bad:
        assert status(**change) == B.MV_ERR_INVALID_ARG, change


def test_values_of_a_call(lib):
    rows = (1 << 29) - 511                                      # blocks of 128: one more than 2^36 - 2^16 values
    for dtype in (B.MV_F32, B.MV_BF16):
        assert lib.mv_f8_encode(P, dtype, 128, rows, 128, 2 * P, 128, 3 * P, 4, None) == B.MV_ERR_INVALID_ARG
        assert lib.mv_f8_decode(2 * P, 128, 3 * P, 4, rows, 128, P, dtype, 128, None) == B.MV_ERR_INVALID_ARG
        # columns: 2^24 tiles of 128 rows, one below the other
        long = (1 << 31) - 127
        assert lib.mv_f8_encode_t(P, dtype, 1, long, 1, 2 * P, 1 << 31, 3 * P, 1 << 24, None) == B.MV_ERR_INVALID_ARG


def test_blocks_of_a_layers_gradients(lib):
    m, n = (1 << 29) - 512, 128                                 # dy's blocks alone would do, with its columns they are too many
    status = lib.mv_f8_linear_grad(P, 1, 2 * P, n, B.MV_F32, 3 * P, 128, 4 * P, 4, m, n, 1, 5 * P, B.MV_F32, 1, 6 * P, B.MV_F32, 1, 7 * P,
                                   1 << 62, None)
    assert status == B.MV_ERR_INVALID_ARG
