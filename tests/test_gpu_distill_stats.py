"""The gradient from a loss's stats is formed from them, whatever the size of a row: with other stats than the row's own it is
the formula's with those."""
import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_distill import TYPES, U, make, scratch_of, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("temperature,soft,hard", [(1.0, 0.7, 0.3), (2.0, 0.7, 0.3), (3.0, 0.7, 0.3), (3.0, 1.0, 0.0), (3.0, 0.0, 1.0)])
@pytest.mark.parametrize("rows,n", [(5, 7), (6500, 60), (9, 1000), (9, 3000), (1010, 2300), (3, 140_000)])
def test_stats_as_they_are_given(rows, n, temperature, soft, hard, src):
    """Largest logits further up and sums that have been multiplied: q and s are smaller by known factors.  With e of a logit's two
    exponentials and their sums each off by a few roundings of an argument below 40, dz is within 400 U of its terms' magnitudes."""
    z, idx, t, label = make(rows, n, 4, src, rows + n, repeats=False)
    at = (z.cuda(), idx.cuda(), t.cuda(), label.cuda(), temperature, soft, hard)
    loss, stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, 3), device="cuda")
    B.mv_distill_loss(*at, loss, scratch_of(rows, n), stats=stats)
    other = stats.clone()
    other[:, 0] += 1.0
    other[:, 1] *= 2.0
    other[:, 2] *= 3.0
    own, dz = torch.zeros((rows, n), device="cuda"), torch.zeros((rows, n), device="cuda")
    B.mv_distill_grad(*at, stats, own)
    B.mv_distill_grad(*at, other, dz)
    s, d = stats.double(), z.double().cuda() - stats[:, :1].double()
    first = soft * temperature * torch.exp(d / temperature) / s[:, 1:2] if soft else torch.zeros_like(d)
    second = hard * torch.exp(d) / s[:, 2:3] if hard else torch.zeros_like(d)
    listed = ((idx >= 0) & (idx < n)).any(1).cuda()[:, None]
    labelled = ((label >= 0) & (label < n)).cuda()[:, None]
    first, second = first * listed, second * labelled
    want = own.double() - first * (1 - torch.exp(torch.tensor(-1.0 / temperature, dtype=torch.float64)) / 2)
    want = want - second * (1 - torch.exp(torch.tensor(-1.0, dtype=torch.float64)) / 3)
    bound = 400 * U * (first + second + own.double().abs()) + 2.0 ** -126 * (1 + temperature)
    assert ((dz.double() - want).abs() <= bound).all(), float(((dz.double() - want).abs() / bound).max())
