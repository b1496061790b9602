"""8-bit products with values at the upper end: the type's largest ones are held as 2^128, beyond fp32 and bf16.  A result that
such a value takes part in is right or not finite, and no other result is touched."""
import numpy as np
import pytest
import torch

import f8_reference as R
from paper_2011_06495_amd import binding as B
from test_gpu_f8_product import TYPES, check, hold, normal, say, scratch_of  # noqa: F401

pytestmark = pytest.mark.gpu


def right_or_lost(out, a, b, dtype, row):
    """Row `row` of a has the value."""
    got = out.float().cpu()
    others = np.delete(np.arange(a.shape[0]), row)
    check(out[torch.from_numpy(others).cuda()], a[others], b, dtype)
    with np.errstate(over="ignore"):
        want = torch.from_numpy((a[row] @ b.T).astype(np.float32)).to(dtype).float()
    size = torch.from_numpy(np.abs(a[row]) @ np.abs(b).T)
    fine = torch.isfinite(got[row])
    off = (got[row].double() - want.double()).abs()
    assert (off[fine] <= (2.0 ** -7 * size)[fine]).all()


# few rows of codes and of values, tiles of each kind
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 40, 300), (12, 300, 4096), (40, 70, 900), (300, 280, 1100), (3600, 3500, 300)])
def test_largest_values(m, n, k, dst):
    rng = np.random.default_rng(m + n)
    x, w = normal(rng, m, k), normal(rng, n, k)
    x[1] = 0.0
    x[1, 130] = np.finfo(np.float32).min
    w[:, 130] = np.where(np.arange(n) % 3 == 0, 0.0, 2.0 ** -40).astype(np.float32)
    w[:, 128:130], w[:, 131:256] = 0.0, 0.0
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(w)
    assert a[1, 130] == -2.0 ** 128
    out = torch.zeros((m, n), dtype=TYPES[dst], device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    right_or_lost(out, a, b, TYPES[dst], 1)
    out.zero_()
    B.mv_f8_linear(torch.from_numpy(x).cuda(), b_codes, b_scales, out, scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k)))
    right_or_lost(out, a, b, TYPES[dst], 1)


@pytest.mark.parametrize("top", [2.0 ** 127, 240.0 * 2.0 ** 120, -247.0 * 2.0 ** 120])
def test_values_below_are_held(top):
    """The largest that is not beyond: products with it are those of what 8 bits hold."""
    m, n, k = 5, 30, 200
    x, w = np.zeros((m, k), np.float32), normal(np.random.default_rng(1), n, k)
    x[:, 7] = top
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(w * np.float32(2.0 ** -20))
    out = torch.zeros((m, n), device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    assert np.array_equal(out.cpu().numpy(), (a @ b.T).astype(np.float32))
