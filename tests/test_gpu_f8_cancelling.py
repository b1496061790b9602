"""bf16 results of few rows are formed without the 8-bit instruction's cut, however long the sums and whichever kernel forms them:
products of 2^12 that cancel, each beside seven of 2^-2 that the cut would take away."""
import numpy as np
import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_f8_product import hold, say, scratch_of  # noqa: F401

pytestmark = pytest.mark.gpu
GROUPS = 256


def cancelling(rows, k, signs):
    """GROUPS groups of eight neighbours, spread over the row: 64 with a sign of its own where asked for, and seven times 1/2; rows
    differ by powers of two."""
    x = np.zeros((rows, k), np.float32)
    for g in range(GROUPS):
        at = (k - 8) // 8 * g // (GROUPS - 1) * 8
        x[:, at] = 64.0 * (-1.0) ** g if signs else 64.0
        x[:, at + 1:at + 8] = 0.5
    return x * np.exp2(np.arange(rows) % 5).astype(np.float32)[:, None]


def wanted(m, n):
    """What is left, 7 * 256 / 4 of each row's powers: whole, and sums on the way below 2^24 quarters."""
    return torch.from_numpy(GROUPS * 7 / 4 * np.outer(np.exp2(np.arange(m) % 5), np.exp2(np.arange(n) % 5))).cuda()


@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(5, 300, 4096), (3, 5, 500_000), (16, 27, 131_072), (1000, 10, 20_000), (16, 2000, 40_000)])
def test_products(m, n, k, dst):
    a_codes, a_scales, a = hold(cancelling(m, k, True))
    b_codes, b_scales, b = hold(cancelling(n, k, False))
    assert np.array_equal(a, cancelling(m, k, True)) and np.array_equal(b, cancelling(n, k, False))
    out = torch.zeros((m, n), dtype=dst, device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    assert torch.equal(out, wanted(m, n).to(dst))
    x = torch.from_numpy(a.astype(np.float32)).cuda()
    if m <= 16:
        out.zero_()
        B.mv_f8_linear(x, b_codes, b_scales, out, scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k)))
        assert torch.equal(out, wanted(m, n).to(dst))


@pytest.mark.parametrize("m,n,k", [(131_072, 16, 27), (100_000, 10, 330)])
def test_weights_gradients(m, n, k):
    """dw alone and beside dx."""
    dy, x = (torch.from_numpy(np.ascontiguousarray(cancelling(rows, m, signs).T)).cuda().bfloat16() for rows, signs in ((n, True), (k, False)))
    wt_codes, wt_scales, _ = hold(np.ones((k, n), np.float32))
    dw, dx = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    scratch = scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k))
    B.mv_f8_linear_grad(x, dy, None, None, None, dw, scratch)
    assert torch.equal(dw, wanted(n, k).bfloat16())
    dw.zero_()
    B.mv_f8_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch)
    assert torch.equal(dw, wanted(n, k).bfloat16())
    # rows of dy: whole numbers of one block whose sum is exact
    assert torch.equal(dx, dy.double().sum(1, keepdim=True).expand(-1, k).bfloat16())
