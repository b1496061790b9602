"""Calls whose workgroups take more than 64 KB of LDS, some of it sized at the launch, captured into a graph and replayed between
eager calls."""
import numpy as np
import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_distill import TYPES, make, say, scratch_of  # noqa: F401
from test_gpu_f8_product import hold, normal

pytestmark = pytest.mark.gpu


def replayed(run, outputs, change):
    run()
    want = [x.clone() for x in outputs]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        for x in outputs:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
        change()
        run()
        want = [x.clone() for x in outputs]


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(1030, 300, 1024), (6, 3000, 4096), (260, 36_000, 4096), (270, 69_000, 40), (300, 16_000, 4096)])
def test_distillation(rows, n, top, src):
    z, idx, t, label = make(rows, n, top, src, rows + n)
    z, at = z.cuda(), (idx.cuda(), t.cuda(), label.cuda(), 3.0, 0.6, 0.4)
    loss, stats, dz, alone = (torch.zeros(s, device="cuda") for s in (rows, (rows, 3), (rows, n), (rows, n)))
    scratch = scratch_of(rows, n)

    def run():
        B.mv_distill_loss(z, *at, loss, scratch, stats=stats, dz=dz)
        B.mv_distill_grad(z, *at, stats, alone)

    replayed(run, (loss, stats, dz, alone), lambda: z.neg_())


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(16, 64, 8192), (8, 100, 8192), (4, 64, 16_384)])
def test_few_rows_of_values(m, n, k, src):
    rng = np.random.default_rng(m + n)
    x = torch.from_numpy(normal(rng, m, k)).cuda().to(TYPES[src])
    c, s, _ = hold(normal(rng, n, k))
    out = torch.zeros((m, n), device="cuda")
    scratch = torch.empty(B.mv_f8_linear_scratch_bytes(m, n, k), dtype=torch.uint8, device="cuda")
    replayed(lambda: B.mv_f8_linear(x, c, s, out, scratch), (out,), lambda: x.neg_())
