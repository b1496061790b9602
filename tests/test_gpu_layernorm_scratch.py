"""A layer norm's gradients write nothing behind the scratch that they ask for."""
import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_layernorm import SHAPES, TYPES, check_backward, make, say, stats_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES + [(100, 300_001), (9, 140_000)])
def test_nothing_behind_the_scratch(rows, n, src):
    x, dy, gamma, _ = make(rows, n, src, "f32", rows + n)
    mean, rstd = stats_of(x)
    need = B.mv_layernorm_scratch_bytes(rows, n)
    room = torch.full((need + (1 << 20),), 0x77, dtype=torch.uint8, device="cuda")
    dx, sums = torch.zeros((rows, n), device="cuda"), torch.zeros((2, n), device="cuda")
    B.mv_layernorm_backward(x.cuda(), dy.cuda(), gamma, mean, rstd, dx, sums[0], sums[1], room[:need])
    check_backward(x, dy, gamma, mean, rstd, dx, sums[0], sums[1])
    assert (room[need:] == 0x77).all()
