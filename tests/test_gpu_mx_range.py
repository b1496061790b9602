"""Microscaled 4-bit values over the whole range of bf16 and by columns: every exponent, ties, denormals, infinities and
NaN, against the definition in numpy (tests/mx_reference.py), exactly."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEAST = {"f32": -149, "bf16": -133}         # exponents of the smallest denormals


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def room(rows, n):
    return (torch.full((rows, B.mv_mx_row_words(n)), 0x5A, dtype=torch.int32, device="cuda"),
            torch.full((rows, B.mv_mx_row_scales(n)), 0x5A, dtype=torch.uint8, device="cuda"))


def check_codes(codes, scales, x):
    want, want_scales = R.encode(x)
    assert np.array_equal(scales.cpu().numpy()[:, : want_scales.shape[1]], want_scales)
    assert np.array_equal(codes.cpu().numpy().view(np.uint32), R.pack(want))
    return R.values(want, want_scales, x.shape[1])


def all_exponents(src):
    """Blocks whose largest value has each exponent of the type: the others at the grid's places and middles (bf16 has the
    bits for them), one unit below, and spread up to twice the power of two, cut at 6."""
    rows = []
    for e in range(LEAST[src], 128):
        top = 2.0 ** e
        step = np.concatenate([np.arange(16) / 16.0, [0.0625, 0.1875, 0.3125, 0.4375, 0.625, 0.875, 1.25]])
        v = np.concatenate([top * step, top * step[16:] * (1.0 - 2.0 ** -8), [1.5 * top, 1.75 * top]])
        rows.append(np.resize(v, 32) * np.where(np.arange(32) % 2, -1, 1))
        rows.append(top * (1.0 + np.arange(32) / 32.0))
        rows.append(np.where(np.arange(32) == 31, -top, 0.0))
    x = np.array(rows)
    most = torch.finfo(TYPES[src]).max
    return torch.from_numpy(np.clip(x, -most, most).astype(np.float32)).to(TYPES[src])


@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_every_exponent_by_rows(src):
    x = all_exponents(src)
    codes, scales = room(*x.shape)
    resid, out = torch.zeros(x.shape, device="cuda"), torch.zeros(x.shape, device="cuda")
    B.mv_mx_encode(x.cuda(), codes, scales, resid=resid)
    x32 = x.float().numpy()
    held = check_codes(codes, scales, x32)
    assert np.array_equal(resid.cpu().numpy().astype(np.float64), x32.astype(np.float64) - held)
    B.mv_mx_decode(codes, scales, out)
    assert np.array_equal(out.cpu().numpy().astype(np.float64), held)
    again = room(*x.shape)
    B.mv_mx_encode(x.cuda(), *again)
    check_codes(*again, x32)


@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_every_exponent_by_columns(src):
    x = all_exponents(src)
    codes, scales = room(*x.shape)
    B.mv_mx_encode_t(x.t().contiguous().cuda(), codes, scales)
    check_codes(codes, scales, x.float().numpy())


@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_nan_and_infinity_by_rows_and_columns(src):
    x = np.ones((5, 200), np.float32)
    x[0, 40], x[1, 5], x[2, 199], x[3, 64], x[3, 96] = np.nan, np.inf, -np.inf, -np.inf, np.nan
    x[4, :32] = np.nan
    d = torch.from_numpy(x).to(TYPES[src])
    lost = np.zeros(x.shape, bool)
    lost[0, 32:64] = lost[1, :32] = lost[2, 192:] = lost[3, 64:128] = lost[4, :32] = True
    codes, scales = room(5, 200)
    resid, out = torch.zeros((5, 200), device="cuda"), torch.zeros((5, 200), device="cuda")
    B.mv_mx_encode(d.cuda(), codes, scales, resid=resid)
    check_codes(codes, scales, x)
    B.mv_mx_decode(codes, scales, out)
    assert np.array_equal(np.isnan(out.cpu().numpy()), lost) and np.array_equal(np.isnan(resid.cpu().numpy()), lost)
    assert (out.cpu().numpy()[~lost] == 1.0).all()
    codes, scales = room(200, 5)
    B.mv_mx_encode_t(d.cuda(), codes, scales)
    check_codes(codes, scales, np.ascontiguousarray(x.T))


@pytest.mark.parametrize("m", [1, 3, 20, 40, 100])
@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_a_layer_of_denormals_and_lost_blocks(src, m):
    """A row of denormals times large weights, one with a NaN, one with an infinity: few rows, which every workgroup quantises
    for itself, and more.  One product a result, so it is exact."""
    n, k = 70, 300
    least = 2.0 ** LEAST[src]
    x = np.zeros((m, k), np.float32)
    x[0, 260:] = least * np.resize([1.0, 3.0, 17.0, -40.0, 5.0], 40)
    x[0, 270] = 47.0 * 2.0 ** -133                  # bf16 has it, too
    if m > 2:
        x[1, 5], x[2, 299] = np.nan, -np.inf
    w = np.zeros((n, k), np.float32)
    w[np.arange(n), 230 + np.arange(n)] = 2.0 ** 120
    codes, scales = room(n, k)
    B.mv_mx_encode(torch.from_numpy(w).cuda(), codes, scales)
    held_w = check_codes(codes, scales, w)
    assert np.array_equal(held_w, w)
    out = torch.full((m, n), 7.5, device="cuda")
    d = torch.from_numpy(x).to(TYPES[src])
    need = B.mv_mx_linear_scratch_bytes(m, n, k)
    B.mv_mx_linear(d.cuda(), codes, scales, out, torch.zeros(need, dtype=torch.uint8, device="cuda"))
    got = out.cpu().numpy()
    clean = [i for i in range(m) if m <= 2 or i not in (1, 2)]
    want = R.held(d.float().numpy()[clean]) @ held_w.T
    assert want[0].any() and np.array_equal(got[clean].astype(np.float64), want)
    if m > 2:
        assert np.isnan(got[1:3]).all()
