"""Layer norm of rows near the ends of fp32's range."""
import math

import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_layernorm import TYPES, check_forward, say  # noqa: F401

pytestmark = pytest.mark.gpu


# rows of a wavefront, of workgroups of each size, and rows beyond the registers
@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n", [5, 64, 1000, 3001, 8192, 16_384, 40_000])
def test_squares_beyond_fp32_have_no_finite_results(n, src, dst):
    """Values around 1e20 and 1e25, whose sum is far inside fp32 and whose squares are not: nothing finite, and the rows beside
    them as they are."""
    gen = torch.Generator().manual_seed(n)
    x = torch.randn((7, n), generator=gen)
    gamma, beta = 1 + 0.3 * torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    x[1] = 1e20 * (1.0 + torch.arange(n) % 2)
    x[4] = 1e25 * (torch.arange(n) % 2)
    x = x.to(TYPES[src])
    y, stats = torch.zeros((7, n), dtype=TYPES[dst], device="cuda"), torch.zeros((2, 7), device="cuda")
    B.mv_layernorm_forward(x.cuda(), gamma.cuda(), beta.cuda(), 1e-5, y, stats[0], stats[1])
    lost, kept = torch.tensor([1, 4]), torch.tensor([0, 2, 3, 5, 6])
    assert not torch.isfinite(y[lost]).any() and not torch.isfinite(stats[1, lost]).any()
    check_forward(x[kept], gamma.cuda(), beta.cuda(), 1e-5, y[kept], stats[0, kept], stats[1, kept])
    # and no gradient of them that looks like one
    dy, dx = torch.randn((7, n), generator=gen).to(TYPES[src]).cuda(), torch.zeros((7, n), dtype=TYPES[dst], device="cuda")
    dgamma, dbeta = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    scratch = torch.empty(B.mv_layernorm_scratch_bytes(7, n), dtype=torch.uint8, device="cuda")
    B.mv_layernorm_backward(x.cuda(), dy, gamma.cuda(), stats[0], stats[1], dx, dgamma, dbeta, scratch)
    assert not torch.isfinite(dx[lost]).any() and torch.isfinite(dx[kept]).all() and torch.isfinite(dbeta).all()


@pytest.mark.parametrize("n", [7, 1000, 40_000])
def test_large_and_small_values_within_fp32(n):
    """Squares' sums just inside fp32, and variances far below eps and above it."""
    gen = torch.Generator().manual_seed(n)
    x = torch.randn((3, n), generator=gen)
    x[0] *= 2.0 ** 63 / math.sqrt(n) / 8
    x[1] *= 2.0 ** -60
    y, stats = torch.zeros((3, n), device="cuda"), torch.zeros((2, 3), device="cuda")
    B.mv_layernorm_forward(x.cuda(), None, None, 1e-5, y, stats[0], stats[1])
    check_forward(x, None, None, 1e-5, y, stats[0], stats[1])
    B.mv_layernorm_forward(x[:2].cuda(), None, None, 0.0, y[:2], stats[0, :2], stats[1, :2])
    check_forward(x[:2], None, None, 0.0, y[:2], stats[0, :2], stats[1, :2])
