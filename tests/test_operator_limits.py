"""How large the operators' arguments may be, by what the header says; all without a device: sizes alone are asked for, or a
call is refused before any device call, and the addresses are made up."""
import ctypes
import os

import pytest

from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import build as mv_build

P = 1 << 20
CHUNKS = (1 << 24) - 1                  # of a list of tensors, at most
F32, BF16 = 8192, 16384                 # elements of a chunk


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        mv_build.build_lib()
    return B.load()


def room(lib, tensors, n_groups=1):
    """Bytes that a list needs, 0 if it is refused; tensors: (elements, group, type)."""
    many = (B.mv_clip_tensor * len(tensors))(*[B.mv_clip_tensor(P, 2 * P, n, g, t, t) for n, g, t in tensors])
    cfg = B.mv_clip_config(ctypes.sizeof(B.mv_clip_config), 0, n_groups, B.MV_NORM_L2, None, 0)
    return lib.mv_clip_workspace_bytes(ctypes.byref(cfg), many, len(tensors))


@pytest.mark.parametrize("dtype,per", [(B.MV_F32, F32), (B.MV_BF16, BF16)])
def test_chunks_of_a_list(lib, dtype, per):
    most = (CHUNKS - 1) * per                                   # one group: one chunk more
    assert room(lib, [(most, 0, dtype)]) > 0
    assert room(lib, [(most + 1, 0, dtype)]) == 0
    assert room(lib, [(most - per, 0, dtype), (1, 0, dtype)]) > 0
    assert room(lib, [(most - per, 0, dtype), (1, 0, dtype), (1, 0, dtype)]) == 0       # each rounded up
    assert room(lib, [(most - 2 * per, 0, dtype), (1, 1, dtype)], 2) > 0
    assert room(lib, [(most - per, 0, dtype), (1, 1, dtype)], 2) == 0                   # and a second group's
    assert room(lib, [(most, 0, dtype), (0, 1, dtype)], 3) > 0                          # groups without elements have none


def test_values_of_a_call(lib):
    rows = (1 << 29) - 511                                      # blocks of 32: one more than 2^34 - 2^14 values
    for dtype in (B.MV_F32, B.MV_BF16):
        assert lib.mv_mx_encode(P, dtype, 32, rows, 32, 2 * P, 4, 3 * P, 4, None, 0, None) == B.MV_ERR_INVALID_ARG
        assert lib.mv_mx_decode(2 * P, 4, 3 * P, 4, rows, 32, P, dtype, 32, None) == B.MV_ERR_INVALID_ARG
        # columns: 2^24 tiles, one below the other
        long = (1 << 31) - 127
        assert lib.mv_mx_encode_t(P, dtype, 1, long, 1, 2 * P, 1 << 28, 3 * P, 1 << 26, None) == B.MV_ERR_INVALID_ARG


def test_blocks_of_a_layers_gradients(lib):
    m, n = (1 << 29) - 512, 32                                  # dy's blocks alone would do, with its columns they are too many
    status = lib.mv_mx_linear_grad(P, 1, 2 * P, n, B.MV_F32, 3 * P, 4, 4 * P, 4, m, n, 1, 5 * P, B.MV_F32, 1, 6 * P, B.MV_F32, 1, 7 * P,
                                   1 << 62, None)
    assert status == B.MV_ERR_INVALID_ARG
