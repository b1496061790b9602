"""Distillation with two exponentials for each logit (both terms and a temperature other than 1 and 2), from fp32 and bf16 logits in
every way that rows are held or stream by, and rows that have no finite result, against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_distill import TYPES, check, make, place, reference, say, scratch_of  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [(96, 10, 4), (6, 100, 200), (4, 1000, 50), (7, 2049, 3), (3, 5000, 100), (4, 16_385, 40), (2, 33_000, 20), (3, 131_073, 33),
          (1, 300_001, 64), (1100, 300, 9), (1010, 2300, 7), (60, 69_000, 12)]


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,n,top", SHAPES)
def test_two_exponentials(rows, n, top, src, dst):
    z, idx, t, label = make(rows, n, top, src, rows + n + top)
    g = torch.randn(rows, generator=torch.Generator().manual_seed(2))
    temperature, soft, hard = 3.0, 0.7, 0.3
    ref = reference(z, idx, t, label, temperature, soft, hard, g)
    zd, td, id_ = place(z, TYPES[src], 1, 3), place(t, TYPES[src], 1, 3), place(idx, torch.int32, 1, 3)
    at = (zd, id_, td, label.cuda(), temperature, soft, hard)
    loss, stats = torch.full((rows + 1,), 7.5, device="cuda"), torch.full((rows + 1, 3), 7.5, device="cuda")
    dz = torch.full((rows + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_distill_loss(*at, loss[:rows], scratch_of(rows, n), stats=stats[:rows], dz=dz[:rows, 1:n + 1], grad=g.cuda())
    check(ref, loss[:rows], dz[:rows, 1:n + 1], stats[:rows])
    alone, again = torch.zeros(rows, device="cuda"), torch.zeros((rows, 3), device="cuda")
    B.mv_distill_loss(*at, alone, scratch_of(rows, n), stats=again)
    check(ref, alone, None, again)
    dz[:rows, 1:n + 1] = 7.5
    assert (dz == 7.5).all() and (loss[rows:] == 7.5).all() and (stats[rows:] == 7.5).all()
    B.mv_distill_grad(*at, again, dz[:rows, 1:n + 1], grad=g.cuda())
    check(ref, None, dz[:rows, 1:n + 1])
    dz[:rows, 1:n + 1] = 7.5
    assert (dz == 7.5).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(4200, 70, 5), (6200, 100, 5), (4200, 2200, 6), (1100, 1500, 30), (520, 20_001, 9), (300, 36_001, 5),
                                        (270, 69_700, 40)])
def test_more_rows_than_run_at_once(rows, n, top, src):
    """Rows that take turns, in place, with both terms at another temperature, and with the second one alone."""
    z, idx, t, label = make(rows, n, top, src, rows + n)
    for soft, hard in ((0.7, 0.3), (0.0, 1.5)):
        ref = reference(z, idx, t, label, 3.0, soft, hard, None)
        loss, d, dz = torch.zeros(rows, device="cuda"), place(z, TYPES[src], 1, 3), torch.zeros((rows, n), device="cuda")
        at = (idx.cuda(), t.cuda(), label.cuda(), 3.0, soft, hard)
        B.mv_distill_loss(d, *at, loss, scratch_of(rows, n), dz=dz)
        check(ref, loss, dz)
        alone, stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, 3), device="cuda")
        B.mv_distill_loss(d, *at, alone, scratch_of(rows, n), stats=stats)
        check(ref, alone)
        B.mv_distill_loss(d, *at, loss, scratch_of(rows, n), dz=d)
        assert torch.equal(d, dz.to(d.dtype))
        d.copy_(z)
        B.mv_distill_grad(d, *at, stats, d)
        dz.copy_(d)
        check(ref, None, dz.to(d.dtype))


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(9, 300, 1024), (1030, 300, 1024), (1030, 2300, 1000), (9, 2300, 4096)])
def test_long_lists_of_two_exponentials(rows, n, top, src):
    """The longest lists that four rows of a workgroup have beside each other, and longer ones."""
    z, idx, t, label = make(rows, n, top, src, top)
    ref = reference(z, idx, t, label, 3.0, 0.7, 0.3, None)
    loss, dz = torch.zeros(rows, device="cuda"), torch.zeros((rows, n), device="cuda")
    B.mv_distill_loss(z.cuda(), idx.cuda(), t.cuda(), label.cuda(), 3.0, 0.7, 0.3, loss, scratch_of(rows, n), dz=dz)
    check(ref, loss, dz)


# rows of a wavefront, of workgroups of each size, whole rows that stream by, ranges of rows
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("rows,n", [(11, 60), (1011, 2300), (11, 5000), (11, 33_000), (1030, 17_000), (11, 140_000)])
def test_rows_without_finite_results(rows, n, temperature, src):
    """All logits masked, one infinite upwards, one NaN (of each sign), and rows without a term with the same: next to
    rows that stay what they are."""
    inf = math.inf
    z, idx, t, label = make(rows, n, 5, src, n + 1, repeats=False)
    label[:] = torch.arange(rows) % n
    idx[:, 0] = (torch.arange(rows) + 20) % n
    lost, none = [1, 3, 4, 6], [7, 8, 9]
    clean = z.clone()
    z[1] = -inf
    z[3, n - 1] = inf
    z[4, n // 2] = math.nan
    z[6, n // 3] = -math.nan
    z[7], z[8, 5], z[9, n - 2] = -inf, inf, math.nan
    idx[none], label[none] = -1, -1
    kept = [r for r in range(rows) if r not in lost and r not in none]
    ref = reference(clean[kept], idx[kept], t[kept], label[kept], temperature, 0.6, 0.4, None)
    loss, stats = torch.full((rows,), 7.5, device="cuda"), torch.zeros((rows, 3), device="cuda")
    dz = torch.full((rows, n), 7.5, dtype=TYPES[src], device="cuda")
    at = (z.cuda(), idx.cuda(), t.cuda(), label.cuda(), temperature, 0.6, 0.4)

    def look(loss, dz):
        if loss is not None:
            assert torch.isnan(loss[lost]).all() and (loss[none] == 0.0).all()
        if dz is not None:
            assert torch.isnan(dz[lost]).all() and (dz[none] == 0.0).all()
        check(ref, loss[kept] if loss is not None else None, dz[kept] if dz is not None else None)

    B.mv_distill_loss(*at, loss, scratch_of(rows, n), dz=dz)
    look(loss, dz)
    loss.fill_(7.5)
    B.mv_distill_loss(*at, loss, scratch_of(rows, n), stats=stats)
    look(loss, None)
    dz.fill_(7.5)
    B.mv_distill_grad(*at, stats, dz)
    look(None, dz)
