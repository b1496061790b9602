"""Layer norm and its gradients against their formulas in 64 bits.

With u = 2^-24, the rounding of one fp32 operation, and L additions on the way of a value into a row's sum (at most 32 of a
thread's own, and of longer rows n / 1024, then 22 over the workgroup): a mean of values v is off by at most (L + 2) u
mean|v|, a variance by (L + 4) u of itself, its root by half of that.  Differences from the mean are rounded once, the product
with rstd and gamma once each, so y = h gamma + beta is off by at most u ((L + 6) (|h| + 1) |gamma| + |beta| + |y|), then by half
a step of its type.  Gradients in the same way, written where they are checked."""
import numpy as np
import pytest
import torch

from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def adds(n):
    return max(56, n // 1024 + 32)


def place(x, dtype, lead=0, extra=0):
    rows, n = x.shape
    flat = torch.full((lead + rows * (n + extra),), 3.0, dtype=dtype, device="cuda")
    out = flat[lead:].view(rows, n + extra)[:, :n]
    out.copy_(x)
    return out


def make(rows, n, src, weights, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, n), generator=gen) * torch.exp(torch.randn((rows, 1), generator=gen)) + torch.randn((rows, 1), generator=gen)
    gamma, beta = 1 + 0.3 * torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    dy = torch.randn((rows, n), generator=gen) * torch.exp(torch.randn((rows, 1), generator=gen))
    return (x.to(TYPES[src]), dy.to(TYPES[src]), gamma.to(TYPES[weights]).cuda() if weights else None,
            beta.to(TYPES[weights]).cuda() if weights else None)


def whole(t, n, other):
    return t.double().cpu() if t is not None else torch.full((n,), other, dtype=torch.float64)


def check_forward(x, gamma, beta, eps, y, mean, rstd):
    x = x.double().cpu()
    n = x.shape[1]
    m = x.mean(1)
    c = x - m[:, None]
    var = c.square().mean(1)
    r = (var + eps) ** -0.5
    h = c * r[:, None]
    g, b = whole(gamma, n, 1.0), whole(beta, n, 0.0)
    want = h * g + b
    L = adds(n)
    bound = U * ((L + 6) * (h.abs() + 1) * g.abs() + b.abs() + want.abs())
    bound += half_step(y.dtype) * (want.abs() + bound)
    off = (y.double().cpu() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())
    if mean is not None:
        assert ((mean.double().cpu() - m).abs() <= U * (2 * m.abs() + (L + 3) * c.abs().mean(1) + L * L * U * x.abs().mean(1))).all()
    if rstd is not None:
        assert ((rstd.double().cpu() - r).abs() <= (L / 2 + 5) * U * r).all()


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 64), (7, 255), (9, 512), (4, 1000), (33, 1024), (3, 2049), (2, 4097), (5, 8192), (2, 8200),
          (1, 16384), (2, 16400), (2, 33_000), (1, 70_001), (1030, 65), (9000, 9), (700, 600), (600, 3000), (2100, 1500), (1100, 6001),
          (520, 12_000), (520, 20_001)]


@pytest.mark.parametrize("src,dst,weights", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"),
                                             ("f32", "bf16", "bf16"), ("f32", "f32", None)])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_forward(rows, n, src, dst, weights):
    x, _, gamma, beta = make(rows, n, src, weights, rows + n)
    for lead, extra in ((0, 0), (1, 3)):
        d = place(x, TYPES[src], lead, extra)
        y = torch.full((rows + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
        stats = torch.full((2, rows + 1), 7.5, device="cuda")
        B.mv_layernorm_forward(d, gamma, beta, 1e-5, y[:rows, 1:n + 1], stats[0, :rows], stats[1, :rows])
        check_forward(x, gamma, beta, 1e-5, y[:rows, 1:n + 1], stats[0, :rows], stats[1, :rows])
        y[:rows, 1:n + 1] = 7.5
        assert (y == 7.5).all() and (stats[:, rows:] == 7.5).all()


@pytest.mark.parametrize("n", [300, 5000, 40_000])
def test_rows_far_from_zero(n):
    """A mean of 30,000 standard deviations: its own rounding is 0.002 of them."""
    x = 30_000.0 + torch.randn((4, n), generator=torch.Generator().manual_seed(n))
    y, mean, rstd = torch.zeros((4, n), device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    B.mv_layernorm_forward(x.cuda(), None, None, 1e-6, y, mean, rstd)
    check_forward(x, None, None, 1e-6, y, mean, rstd)


@pytest.mark.parametrize("n", [200, 3000, 40_000])
def test_lost_rows_are_alone(n):
    x = torch.randn((6, n), generator=torch.Generator().manual_seed(1))
    good = x.clone()
    x[1, n // 2], x[4, 0] = float("nan"), float("inf")
    y, mean, rstd = torch.zeros((6, n), device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda")
    B.mv_layernorm_forward(x.cuda(), None, None, 1e-5, y, mean, rstd)
    lost = torch.tensor([1, 4])
    kept = torch.tensor([0, 2, 3, 5])
    assert torch.isnan(y[lost]).all() and not torch.isfinite(mean[lost]).any()
    check_forward(good[kept], None, None, 1e-5, y[kept], mean[kept], rstd[kept])


def test_equal_values():
    for n in (1, 5, 1000, 40_000):
        x = torch.full((3, n), 5.0, device="cuda")
        x[1] = 0.1
        y, rstd = torch.ones((3, n), device="cuda"), torch.zeros(3, device="cuda")
        B.mv_layernorm_forward(x, None, None, 1e-5, y, None, rstd)
        # the rest of a mean's rounding, at most L u |x|, times rstd, below 317
        assert (y.abs() <= adds(n) * U * 5.0 * 317).all() and ((rstd - 1e-5 ** -0.5).abs() <= 0.01).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("n", [77, 3000, 20_000, 40_000])
def test_in_place(n, src):
    x, dy, gamma, beta = make(9, n, src, "f32", n)
    d, y = place(x, TYPES[src], 1, 5), torch.zeros((9, n), dtype=TYPES[src], device="cuda")
    mean, rstd = torch.zeros(9, device="cuda"), torch.zeros(9, device="cuda")
    B.mv_layernorm_forward(d, gamma, beta, 1e-5, y, mean, rstd)
    B.mv_layernorm_forward(d, gamma, beta, 1e-5, d)
    assert torch.equal(d, y)
    scratch = torch.empty(B.mv_layernorm_scratch_bytes(9, n), dtype=torch.uint8, device="cuda")
    xd, dx, sums, more = x.cuda(), torch.zeros((9, n), dtype=TYPES[src], device="cuda"), torch.zeros((2, n), device="cuda"), torch.zeros((2, n), device="cuda")
    B.mv_layernorm_backward(xd, dy.cuda(), gamma, mean, rstd, dx, sums[0], sums[1], scratch)
    for over in ("dy", "x"):
        a, g = xd.clone(), dy.cuda()
        B.mv_layernorm_backward(a, g, gamma, mean, rstd, g if over == "dy" else a, more[0], more[1], scratch)
        assert torch.equal(g if over == "dy" else a, dx) and torch.equal(more, sums)


def check_backward(x, dy, gamma, mean, rstd, dx, dgamma, dbeta):
    """h is off by 2 u |h|, d by u |d|; their means by (L + 2) u mean|d| and (L + 6) u mean|d h|; dx has three more roundings.
    Sums over rows: R of a workgroup's own, 48 when its sums are joined, four where its wavefronts' are."""
    x, dy, mean, rstd = (t.double().cpu() for t in (x, dy, mean, rstd))
    rows, n = x.shape
    h = (x - mean[:, None]) * rstd[:, None]
    d = dy * whole(gamma, n, 1.0)
    along, both = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
    if dx is not None:
        want = rstd[:, None] * (d - along - h * both)
        bound = U * rstd[:, None] * ((adds(n) + 8) * (d.abs().mean(1, keepdim=True) + h.abs() * (d * h).abs().mean(1, keepdim=True)) +
                                     6 * (d.abs() + along.abs() + (h * both).abs()))
        bound += half_step(dx.dtype) * (want.abs() + bound)
        off = (dx.double().cpu() - want).abs()
        assert (off <= bound).all(), float((off / bound).max())
    R = rows // 8 + 64
    if dgamma is not None:
        off, bound = (dgamma.double().cpu() - (dy * h).sum(0)).abs(), (R + 3) * U * (dy * h).abs().sum(0)
        assert (off <= bound).all(), float((off / bound).max())
    if dbeta is not None:
        off, bound = (dbeta.double().cpu() - dy.sum(0)).abs(), R * U * dy.abs().sum(0)
        assert (off <= bound).all(), float((off / bound).max())


def stats_of(x):
    x = x.double()
    return x.mean(1).float().cuda(), ((x - x.mean(1, keepdim=True)).square().mean(1) + 1e-5).rsqrt().float().cuda()


@pytest.mark.parametrize("src,dst,weights", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"),
                                             ("f32", "bf16", None)])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_backward(rows, n, src, dst, weights):
    x, dy, gamma, _ = make(rows, n, src, weights, rows + n)
    mean, rstd = stats_of(x)
    scratch = torch.full((B.mv_layernorm_scratch_bytes(rows, n),), 0x77, dtype=torch.uint8, device="cuda")
    for lead, extra in ((0, 0), (1, 3)):
        a, g = place(x, TYPES[src], lead, extra), place(dy, TYPES[src], lead, extra)
        dx = torch.full((rows + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
        sums = torch.full((2, n + 1), 7.5, device="cuda")
        B.mv_layernorm_backward(a, g, gamma, mean, rstd, dx[:rows, 1:n + 1], sums[0, :n], sums[1, :n], scratch)
        check_backward(x, dy, gamma, mean, rstd, dx[:rows, 1:n + 1], sums[0, :n], sums[1, :n])
        keep = dx[:rows, 1:n + 1].clone()
        dx[:rows, 1:n + 1] = 7.5
        assert (dx == 7.5).all() and (sums[:, n:] == 7.5).all()
    # each alone
    alone, one, two = torch.zeros_like(keep), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    B.mv_layernorm_backward(a, g, gamma, mean, rstd, alone, None, None, scratch)
    B.mv_layernorm_backward(a, g, gamma, mean, rstd, None, one, None, scratch)
    B.mv_layernorm_backward(a, g, gamma, mean, rstd, None, None, two, scratch)
    assert torch.equal(alone, keep) and torch.equal(one, sums[0, :n]) and torch.equal(two, sums[1, :n])


def test_backward_against_differences():
    """The loss sum(dy y) of the forward pass in 64 bits, on both sides of a value."""
    rows, n, eps = 5, 300, 1e-3
    x, dy, gamma, beta = (t.double() if t.dim() == 2 else t.double().cpu() for t in make(rows, n, "f32", "f32", 3))

    def loss(x, gamma, beta):
        c = x - x.mean(1, keepdim=True)
        return float((dy * (c * (c.square().mean(1, keepdim=True) + eps).rsqrt() * gamma + beta)).sum())

    y, mean, rstd = torch.zeros((rows, n), device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    B.mv_layernorm_forward(x.float().cuda(), gamma.float().cuda(), beta.float().cuda(), eps, y, mean, rstd)
    dx, dgamma, dbeta = torch.zeros((rows, n), device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    scratch = torch.empty(B.mv_layernorm_scratch_bytes(rows, n), dtype=torch.uint8, device="cuda")
    B.mv_layernorm_backward(x.float().cuda(), dy.float().cuda(), gamma.float().cuda(), mean, rstd, dx, dgamma, dbeta, scratch)
    step = 1e-4
    for i, j in ((0, 0), (3, 17), (4, 299)):
        for what, grad in ((x, dx[i, j]), (gamma, dgamma[j]), (beta, dbeta[j])):
            at = (i, j) if what.dim() == 2 else (j,)
            keep = float(what[at])
            what[at] = keep + step
            up = loss(x, gamma, beta)
            what[at] = keep - step
            down = loss(x, gamma, beta)
            what[at] = keep
            # a difference's own error: step^2 and 64-bit rounding over the step
            assert abs((up - down) / (2 * step) - float(grad)) <= 1e-5 * (1 + abs(float(grad)))


def test_equal_results_each_time_and_in_a_graph():
    for rows, n in ((5, 100), (2000, 700), (40, 9000), (3, 40_000)):
        x, dy, gamma, beta = make(rows, n, "bf16", "f32", n)
        x, dy = x.cuda(), dy.cuda()
        y, dx = torch.zeros((rows, n), device="cuda"), torch.zeros((rows, n), device="cuda")
        mean, rstd, sums = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros((2, n), device="cuda")
        scratch = torch.empty(B.mv_layernorm_scratch_bytes(rows, n), dtype=torch.uint8, device="cuda")

        def run(stream=None):
            B.mv_layernorm_forward(x, gamma, beta, 1e-5, y, mean, rstd, stream=stream)
            B.mv_layernorm_backward(x, dy, gamma, mean, rstd, dx, sums[0], sums[1], scratch, stream=stream)

        run()
        want = [t.clone() for t in (y, mean, rstd, dx, sums)]
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        for t in (y, mean, rstd, dx, sums):
            t.zero_()
        torch.cuda.synchronize()
        run(other)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd, dx, sums), want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for _ in range(3):
            for t in (y, mean, rstd, dx, sums):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd, dx, sums), want))
            x.neg_()
            run()
            want = [t.clone() for t in (y, mean, rstd, dx, sums)]


def test_many_values_beyond_32_bits():
    """2^32 + 2^18 values in rows of 2^16: the last rows against rows of their own."""
    rows, n = (1 << 16) + 4, 1 << 16
    x = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda").normal_()
    y, mean, rstd = torch.empty_like(x), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    B.mv_layernorm_forward(x, None, None, 1e-5, y, mean, rstd)
    check_forward(x[-3:], None, None, 1e-5, y[-3:], mean[-3:], rstd[-3:])


def test_python_refusals():
    x, y, v = torch.zeros((4, 100), device="cuda"), torch.zeros((4, 100), device="cuda"), torch.ones(100, device="cuda")
    r = torch.zeros(4, device="cuda")
    scratch = torch.empty(B.mv_layernorm_scratch_bytes(4, 100), dtype=torch.uint8, device="cuda")
    for bad in (lambda: B.mv_layernorm_forward(x.double(), v, v, 1e-5, y), lambda: B.mv_layernorm_forward(x, v[:99], v, 1e-5, y),
                lambda: B.mv_layernorm_forward(x, v, v.bfloat16(), 1e-5, y), lambda: B.mv_layernorm_forward(x, v.cpu(), v, 1e-5, y),
                lambda: B.mv_layernorm_forward(x, v, v, 1e-5, y[:3]), lambda: B.mv_layernorm_forward(x, v, v, 1e-5, y, r[:3]),
                lambda: B.mv_layernorm_forward(x.t(), v, v, 1e-5, y.t()),
                lambda: B.mv_layernorm_backward(x, y.bfloat16(), v, r, r, y, v, v, scratch),
                lambda: B.mv_layernorm_backward(x, y, v, r[:3], r, y, v, v, scratch),
                lambda: B.mv_layernorm_backward(x, y, v, r, r, y, v[:99], v, scratch),
                lambda: B.mv_layernorm_backward(x, y, v, r, r, y, v, v, scratch.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.mv_layernorm_forward(x, v, v, -1.0, y), lambda: B.mv_layernorm_backward(x, y, v, r, r, y, v, v, scratch[:64]),
                lambda: B.mv_layernorm_backward(x, y, v, r, None, y, v, v, scratch),
                lambda: B.mv_layernorm_backward(x, y, v, r, r, None, None, None, scratch)):
        with pytest.raises(B.MvError) as e:
            bad()
        assert e.value.status == B.MV_ERR_INVALID_ARG
