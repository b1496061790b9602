"""Two clipping handles at work at once, on two streams: neither finds the whole GPU free."""
import time

import pytest
import torch

from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

GROUPS, VALUES = 4, 11_173_962          # 45 MB a group, of the 57 that a launch's workgroups hold


def test_two_handles_on_two_streams():
    """Results are those of each alone.  Time: at most about half a millisecond of waiting for each of the eight groups, and
    two readings more of 0.36 GB by few workgroups, a millisecond; ten are allowed for both together."""
    sides = []
    for i in range(2):
        x = torch.randn((GROUPS, VALUES), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")
        out, norms = torch.zeros_like(x), torch.zeros(GROUPS, device="cuda")
        h = B.mv_clip_begin(list(x), out=list(out), groups=range(GROUPS))
        B.mv_clip_grads(h, 1000.0, norms)
        torch.cuda.synchronize()
        sides.append((h, x, out, norms, out.clone(), norms.clone(), torch.cuda.Stream()))      # the handle has x's address
    took = []
    for _ in range(6):
        for _, _, out, norms, _, _, _ in sides:
            out.zero_()
            norms.zero_()
        torch.cuda.synchronize()
        at = time.perf_counter()
        for h, _, _, norms, _, _, stream in sides:
            B.mv_clip_grads(h, 1000.0, norms, stream=stream)
        torch.cuda.synchronize()
        took.append(time.perf_counter() - at)
        for _, _, out, norms, want, want_norms, _ in sides:
            assert torch.equal(norms, want_norms) and torch.equal(out, want)
    print(["%.2f ms" % (1e3 * t) for t in took], flush=True)
    for side in sides:
        B.mv_clip_end(side[0])
        B.mv_clip_release(side[0])
    assert max(took[1:]) < 10e-3, took
