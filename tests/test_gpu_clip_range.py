"""Norms at the upper end of fp32, in all three ways that a group is clipped: by one workgroup, read once, and read twice."""
import pytest
import torch

from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [100, 1_000_000, 31_000_000])
def test_norms_around_the_largest_fp32(n, dtype):
    """Values of 2^126, n of them: 2^126 sqrt(n) is beyond fp32 from n = 4 on, and then the factor is 0 and so is the result; the
    largest magnitude is not, and clips as ever; neither is the norm of values of 2^100."""
    for value, kind, norm in ((2.0 ** 126, B.MV_NORM_L2, float("inf")), (2.0 ** 126, B.MV_NORM_MAX, 2.0 ** 126),
                              (2.0 ** 100, B.MV_NORM_L2, 2.0 ** 100 * n ** 0.5)):
        x = torch.full((n,), value, device="cuda").to(dtype)
        x[n // 2] = -value
        out = torch.full((n,), 7.5, dtype=dtype, device="cuda")
        norms, coefs = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        h = B.mv_clip_begin([x], out=[out], norm=kind)
        B.mv_clip_grads(h, 2.0 ** 90, norms, coefs)
        torch.cuda.synchronize()
        B.mv_clip_end(h)
        B.mv_clip_release(h)
        got = float(norms[0])
        # the root of an exact sum, rounded in fp64 and to fp32
        assert got == norm or abs(got - norm) <= norm * 2.0 ** -23
        want = torch.tensor([2.0 ** 90]) / (norms.cpu() + torch.tensor([1e-6]))
        assert torch.equal(coefs.cpu(), want) and (float(want) == 0.0) == (norm == float("inf"))
        assert torch.equal(out, (x.float() * coefs).to(dtype))
        if norm == float("inf"):
            assert not out.any()
