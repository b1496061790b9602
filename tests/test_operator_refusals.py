"""Arguments that the clipping and 4-bit calls refuse, all before any device call: the addresses here are made up."""
import ctypes
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


def test_struct_layouts():
    assert ctypes.sizeof(B.mv_clip_tensor) == 32 and B.mv_clip_tensor.group.offset == 24
    assert ctypes.sizeof(B.mv_clip_config) == 32 and B.mv_clip_config.workspace.offset == 16


def clip_config(**change):
    at = dict(struct_size=ctypes.sizeof(B.mv_clip_config), device=0, n_groups=2, norm=B.MV_NORM_L2, workspace=None, workspace_bytes=0)
    at.update(change)
    return B.mv_clip_config(*at.values())


def clip_tensor(**change):
    at = dict(src=P, dst=2 * P, numel=100, group=0, src_dtype=B.MV_F32, dst_dtype=B.MV_F32)
    at.update(change)
    return B.mv_clip_tensor(*at.values())


def refused(lib, cfg, tensors):
    many = (B.mv_clip_tensor * max(1, len(tensors)))(*tensors)
    h = ctypes.c_void_p()
    status = lib.mv_clip_begin(ctypes.byref(cfg), many, len(tensors), ctypes.byref(h))
    assert not h.value
    return status == B.MV_ERR_INVALID_ARG and lib.mv_clip_workspace_bytes(ctypes.byref(cfg), many, len(tensors)) == 0


def test_clip_lists(lib):
    good = (B.mv_clip_tensor * 2)(clip_tensor(), clip_tensor(src=0, dst=0, numel=0, group=1))
    size = lib.mv_clip_workspace_bytes(ctypes.byref(clip_config()), good, 2)
    assert 0 < size < 1 << 20
    for change in (dict(struct_size=8), dict(device=-1), dict(n_groups=0), dict(n_groups=65536), dict(norm=2)):
        assert refused(lib, clip_config(**change), [clip_tensor()]), change
    for change in (dict(src=0), dict(src=P + 2), dict(dst=2 * P + 1), dict(numel=-1), dict(numel=(1 << 40) + 1), dict(group=2),
                   dict(group=-1), dict(src_dtype=2), dict(dst_dtype=-1), dict(src=P + 1, src_dtype=B.MV_BF16),
                   dict(dst=P, dst_dtype=B.MV_BF16), dict(numel=1 << 40)):
        assert refused(lib, clip_config(), [clip_tensor(), clip_tensor(**change)]), change
    assert refused(lib, clip_config(), [])
    assert refused(lib, clip_config(), [clip_tensor(), clip_tensor(dst=0)])          # some written, some not
    assert lib.mv_clip_begin(None, good, 2, ctypes.byref(ctypes.c_void_p())) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_begin(ctypes.byref(clip_config()), None, 2, ctypes.byref(ctypes.c_void_p())) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_begin(ctypes.byref(clip_config()), good, 2, None) == B.MV_ERR_INVALID_ARG
    for change in (dict(workspace=P, workspace_bytes=size - 1), dict(workspace=P + 64, workspace_bytes=1 << 20)):
        assert lib.mv_clip_begin(ctypes.byref(clip_config(**change)), good, 2, ctypes.byref(ctypes.c_void_p())) == B.MV_ERR_INVALID_ARG


def test_clip_null_handles(lib):
    assert lib.mv_clip_norms(None, P, None) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_grads(None, 1.0, P, None, None) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_bind(None, P, P, None) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_set_spin_limit(None, 1) == B.MV_ERR_INVALID_ARG
    assert lib.mv_clip_end(None) == B.MV_ERR_INVALID_ARG
    lib.mv_clip_release(None)


def test_mx_sizes(lib):
    assert [B.mv_mx_row_words(n) for n in (0, 1, 32, 33, 100, (1 << 31) - 1, 1 << 31)] == [0, 4, 4, 8, 16, 1 << 28, 0]
    assert [B.mv_mx_row_scales(n) for n in (0, 1, 32, 128, 129, (1 << 31) - 1, -5)] == [0, 4, 4, 4, 8, 1 << 26, 0]
    for f in (B.mv_mx_product_scratch_bytes, B.mv_mx_linear_scratch_bytes, B.mv_mx_linear_grad_scratch_bytes):
        assert f(0, 1, 1) == 0 and f(1, 1 << 31, 1) == 0 and f(1, 1, -1) == 0
    assert B.mv_mx_linear_grad_scratch_bytes(100, 100, 100) > 0


# every call with good arguments by name, in the order of the C declaration
CALLS = {
    "mv_mx_encode": dict(vals=P, dtype=0, ld_vals=100, rows=4, n=100, codes=2 * P, ld_words=16, scales=3 * P, ld_scales=4, resid=4 * P,
                         ld_resid=100, stream=None),
    "mv_mx_encode_t": dict(vals=P, dtype=0, ld_vals=100, rows=4, n=100, codes=2 * P, ld_words=4, scales=3 * P, ld_scales=4, stream=None),
    "mv_mx_decode": dict(codes=2 * P, ld_words=16, scales=3 * P, ld_scales=4, rows=4, n=100, out=P, dtype=0, ld_out=100, stream=None),
    "mv_mx_aggregate": dict(codes=2 * P, ld_words=16, scales=3 * P, ld_scales=4, rows=4, n=100, weights=P, agg=4 * P, stream=None),
    "mv_mx_product": dict(a_codes=P, ld_aw=16, a_scales=2 * P, ld_as=4, b_codes=3 * P, ld_bw=16, b_scales=4 * P, ld_bs=4, m=4, n=100,
                          k=100, c=5 * P, c_dtype=0, ld_c=100, scratch=6 * P, scratch_bytes=1 << 20, stream=None),
    "mv_mx_linear": dict(x=P, x_dtype=0, ld_x=100, w_codes=3 * P, ld_words=16, w_scales=4 * P, ld_scales=4, m=40, n=100, k=100, y=5 * P,
                         y_dtype=0, ld_y=100, scratch=6 * P, scratch_bytes=1 << 20, stream=None),
    "mv_mx_linear_grad": dict(x=P, ld_x=100, dy=2 * P, ld_dy=100, dtype=0, wt_codes=3 * P, ld_words=16, wt_scales=4 * P, ld_scales=4,
                              m=40, n=100, k=100, dx=5 * P, dx_dtype=0, ld_dx=100, dw=7 * P, dw_dtype=0, ld_dw=100, scratch=6 * P,
                              scratch_bytes=1 << 20, stream=None),
}
POINTERS = {"vals": 2, "codes": 8, "scales": 2, "out": 2, "agg": 2, "a_codes": 8, "a_scales": 2, "b_codes": 8, "b_scales": 2, "c": 2,
            "x": 2, "w_codes": 8, "w_scales": 2, "y": 2, "dy": 2, "wt_codes": 8, "wt_scales": 2}
OPTIONAL = {"resid": 2, "weights": 2, "dx": 2, "dw": 2}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_mx_arguments(lib, name):
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
            if ld in ("ld_words", "ld_scales", "ld_aw", "ld_as", "ld_bw", "ld_bs"):
                bad += [{ld: good[ld] + 2}]
        if ld.endswith("dtype"):
            bad += [{ld: 2}, {ld: -1}]
    if name in ("mv_mx_linear", "mv_mx_linear_grad"):
        bad += [{"scratch": 0}, {"scratch": good["scratch"] + 8}, {"scratch_bytes": 64}]
    if name == "mv_mx_linear_grad":
        bad += [{"dx": 0, "dw": 0}]
    if name == "mv_mx_encode":
        bad += [{"resid": good["vals"], "dtype": B.MV_BF16}, {"resid": good["vals"], "ld_resid": 104}]
    if name in ("mv_mx_encode", "mv_mx_decode"):
        bad += [{"rows": (1 << 31) - 1, "n": 1 << 20, "ld_vals" if "vals" in good else "ld_out": 1 << 20, "ld_resid": 1 << 20,
                 "ld_words": 1 << 17, "ld_scales": 1 << 15}]
    for change in bad:
        change = {k: v for k, v in change.items() if k in good}
        assert status(**change) == B.MV_ERR_INVALID_ARG, change
