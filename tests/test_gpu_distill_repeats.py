"""Lists that name coordinates many times: what they come to, and that a list costs as its length, not as its square."""
import time

import pytest
import torch

from paper_2011_06495_amd import binding as B
from test_gpu_distill import TYPES, check, make, reference, scratch_of, say  # noqa: F401

pytestmark = pytest.mark.gpu


def crowded(idx, n, how):
    """The list's coordinates gathered on a few."""
    top = idx.shape[1]
    j = torch.arange(top)
    if how == "one":
        return torch.full_like(idx, n // 2)
    if how == "few":                                    # some coordinates of every stretch, entries that are none between them
        few = (j * 7 % 5) * max(1, n // 6) % n
        return torch.where(j % 11 == 3, -1, few).to(torch.int32).expand_as(idx).contiguous()
    if how == "pairs":                                  # each coordinate in both halves
        return torch.where(j < top // 2, idx, idx.roll(top // 2, 1))
    return torch.where(j % 3 == 0, idx, n - 1).to(torch.int32)       # some of their own, the others the last one


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["one", "few", "pairs", "some"])
@pytest.mark.parametrize("rows,n,top", [(5, 40, 70), (1100, 200, 64), (6, 3000, 257), (1010, 2300, 130), (4, 36_000, 4096), (5, 70_000, 300),
                                        (3, 140_000, 1000)])
def test_repeats(rows, n, top, how, src):
    z, idx, t, label = make(rows, n, top, src, rows + n + top, repeats=False)
    idx = crowded(idx, n, how)
    label[::2] = idx[::2, 0]
    ref = reference(z, idx, t, label, 3.0, 0.7, 0.3, None)
    loss, dz, stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, n), device="cuda"), torch.zeros((rows, 3), device="cuda")
    at = (z.cuda(), idx.cuda(), t.cuda(), label.cuda(), 3.0, 0.7, 0.3)
    B.mv_distill_loss(*at, loss, scratch_of(rows, n), stats=stats, dz=dz)
    check(ref, loss, dz)
    first = dz.clone()
    B.mv_distill_loss(*at, loss, scratch_of(rows, n), dz=dz)
    assert torch.equal(dz, first)
    B.mv_distill_grad(*at, stats, dz)
    check(ref, None, dz)


@pytest.mark.parametrize("rows,n,top", [(64, 300, 1024), (64, 5000, 4096), (64, 36_000, 4096)])
def test_a_list_costs_as_its_length(rows, n, top):
    """A list that is filled up with one coordinate and -infinity, and one that names one coordinate only, against one that names
    each coordinate once or is filled up with -1: a hundred times their time leaves room for anything but a square."""
    z = torch.randn((rows, n), device="cuda")
    t = torch.randn((rows, top), device="cuda")
    own = torch.full((rows, top), -1, dtype=torch.int32, device="cuda")
    own[:, : min(n, top)] = torch.arange(min(n, top), dtype=torch.int32, device="cuda")
    filled, low = torch.zeros_like(own), t.clone()
    filled[:, :16] = own[:, :16]
    low[:, 16:] = -float("inf")
    loss, dz = torch.zeros(rows, device="cuda"), torch.zeros((rows, n), device="cuda")

    def took(idx, t):
        best = float("inf")
        for _ in range(4):
            torch.cuda.synchronize()
            start = time.perf_counter()
            B.mv_distill_loss(z, idx, t, None, 2.0, 1.0, 0.0, loss, scratch_of(rows, n), dz=dz)
            torch.cuda.synchronize()
            best = min(best, time.perf_counter() - start)
        return best

    plain = took(own, t)
    for name, spent in (("filled up", took(filled, low)), ("one coordinate", took(torch.full_like(own, 7), t))):
        print("%s: %.1f us, each once %.1f us" % (name, spent * 1e6, plain * 1e6), flush=True)
        assert spent <= 100 * plain
