"""8-bit products of few rows along a long k are split over the units: their splits' sums pass through the scratch, and the
results are held to the bounds of the products' own tests."""
import numpy as np
import pytest
import torch

import f8_reference as R
from paper_2011_06495_amd import binding as B
from test_gpu_f8_product import TYPES, check, hold, normal, say, scratch_of  # noqa: F401

pytestmark = pytest.mark.gpu


def split(scratch, size):
    """Whether the last `size` bytes, the splits' sums, have been written."""
    assert size > 0
    return bool((scratch[scratch.numel() - size:] != 0x77).any())


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 5, 3_000_001), (1, 1, 1_000_000), (16, 27, 131_072), (330, 10, 100_003), (1, 512, 70_000),
                                   (16, 1000, 16_500), (2000, 7, 40_000)])
def test_product(m, n, k, dst):
    rng = np.random.default_rng(m + n + k)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    need = B.mv_f8_product_scratch_bytes(m, n, k)
    scratch = scratch_of(need)
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out[:m, 1:n + 1], scratch)
    check(out[:m, 1:n + 1], a, b, TYPES[dst])
    out[:m, 1:n + 1] = 7.5
    assert (out == 7.5).all() and split(scratch, need)


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 64, 100_000), (4, 500, 30_001), (16, 64, 12_000)])
def test_linear(m, n, k, src):
    rng = np.random.default_rng(m + n + k)
    x = torch.from_numpy(normal(rng, m, k)).cuda().to(TYPES[src])
    w_codes, w_scales, w = hold(normal(rng, n, k))
    out = torch.zeros((m, n), device="cuda")
    scratch = scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k))
    B.mv_f8_linear(x, w_codes, w_scales, out, scratch)
    check(out, R.held(x.float().cpu().numpy()), w, torch.float32)
    assert split(scratch, B.mv_f8_product_scratch_bytes(m, n, k))


def test_weights_gradient_of_few_channels():
    """A first layer's: 27 inputs and 16 outputs of each of 131,072 places."""
    m, n, k = 131_072, 16, 27
    rng = np.random.default_rng(3)
    x, dy = (torch.from_numpy(normal(rng, m, width)).cuda().bfloat16() for width in (k, n))
    dw = torch.zeros((n, k), device="cuda")
    scratch = scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k))
    B.mv_f8_linear_grad(x, dy, None, None, None, dw, scratch)
    held = [R.held(np.ascontiguousarray(v.float().cpu().numpy().T)) for v in (dy, x)]
    check(dw, *held, torch.float32)
    # dw's sums lie behind the quantised matrices, before dx's
    assert split(scratch, B.mv_f8_product_scratch_bytes(n, k, m) + B.mv_f8_product_scratch_bytes(m, k, n))
