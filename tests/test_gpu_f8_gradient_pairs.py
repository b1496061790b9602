"""Both gradients of a layer in 8 bits in one call, in every way that two products share launches, against numpy in 64 bits
with the bounds of the products' own tests: results of both types, tiles of both sizes, one buffer and two, sums of both
products split and joined together."""
import numpy as np
import pytest
import torch

import f8_reference as R
from paper_2011_06495_amd import binding as B
from test_gpu_f8_product import TYPES, check, hold, normal, say, scratch_of  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(m, n, k, dx_type, dw_type, src="bf16"):
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    x, dy = (torch.from_numpy(normal(rng, m, width)).cuda().to(TYPES[src]) for width in (k, n))
    wt_codes, wt_scales, wt = hold(normal(rng, k, n))
    dx = torch.full((m + 1, k + 3), 7.5, dtype=TYPES[dx_type], device="cuda")
    dw = torch.full((n + 1, k + 5), 7.5, dtype=TYPES[dw_type], device="cuda")
    B.mv_f8_linear_grad(x, dy, wt_codes, wt_scales, dx[:m, 1:k + 1], dw[:n, 3:k + 3], scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k)))
    x32, dy32 = x.float().cpu().numpy(), dy.float().cpu().numpy()
    check(dx[:m, 1:k + 1], R.held(dy32), wt, TYPES[dx_type])
    check(dw[:n, 3:k + 3], R.held(np.ascontiguousarray(dy32.T)), R.held(np.ascontiguousarray(x32.T)), TYPES[dw_type])
    dx[:m, 1:k + 1], dw[:n, 3:k + 3] = 7.5, 7.5
    assert (dx == 7.5).all() and (dw == 7.5).all()


@pytest.mark.parametrize("both", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [
    (4900, 512, 4608),      # one product alone would take the larger tiles
    (1000, 1000, 1000),     # both sums are split, and joined in one launch
    (1001, 999, 1003),
    (500, 400, 5000),       # few steps of both and more tiles than units: one buffer
    (300, 2000, 4000),
    (500, 10, 300),         # a product of few rows beside one in tiles
    (12, 3000, 1000),
    (2000, 12, 2500),       # and in launches of their own
    (9, 14, 300),           # few rows of both
])
def test_both_types(m, n, k, both):
    gradients(m, n, k, both, both)


@pytest.mark.parametrize("m,n,k", [
    (2100, 2200, 3700),     # the larger tiles for both products
    (512, 500, 25_000),     # and with few steps
])
def test_larger_tiles_for_both(m, n, k):
    gradients(m, n, k, "bf16", "bf16")


@pytest.mark.parametrize("dx,dw", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,n,k", [(1000, 1000, 1000), (500, 10, 300), (2100, 2200, 600)])
def test_types_of_their_own(m, n, k, dx, dw):
    gradients(m, n, k, dx, dw, "f32")
