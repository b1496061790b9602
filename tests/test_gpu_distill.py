"""Distillation from a teacher's top logits against its formulas in 64 bits.

With u = 2^-24 and a = (z - largest) / T: the argument of an exponential has three roundings, 4 u |a| with some room, and the
function a few u, so an exponential is off by (4 |a| + 4) u of itself; a sum of them by their mean |a| in the same way, and by
L u, L the additions on a value's way into it (at most 128 of a thread's own in registers and 22 over the workgroup; of
longer rows a thread's share, with a rescaling where its largest moves).  The same holds for p, whose sum has its log taken
and off.  Every bound below is made of these."""
import math

import pytest
import torch

from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def place(x, dtype, lead=0, extra=0):
    rows, n = x.shape
    flat = torch.full((lead + rows * (n + extra),), 3, dtype=dtype, device="cuda")
    out = flat[lead:].view(rows, n + extra)[:, :n]
    out.copy_(x)
    return out


def make(rows, n, top, src, seed, repeats=True):
    """Logits, a list with entries that are none, coordinates named twice and thrice, labels of which some are none."""
    gen = torch.Generator().manual_seed(seed)
    z = 2.0 * torch.randn((rows, n), generator=gen)
    t = 3.0 * torch.randn((rows, top), generator=gen)
    idx = torch.stack([torch.randperm(n, generator=gen)[:top] if top <= n else torch.randint(0, n, (top,), generator=gen)
                       for _ in range(rows)]).reshape(rows, top)
    if top > 2:
        idx[torch.rand((rows, top), generator=gen) < 0.1] = -1
        idx[:, 1] = torch.tensor([-5, n, 2 ** 31 - 1])[torch.arange(rows) % 3]
        if repeats:
            idx[:, top - 1] = idx[:, 0]
            idx[:, top // 2] = idx[:, 0]
    label = torch.randint(0, n, (rows,), generator=gen)
    if top:
        label[::3] = idx[::3, 0]                        # sometimes what the teacher lists
    label[1::4] = torch.tensor([-1, n, -100])[torch.arange(len(label[1::4])) % 3]
    return z.to(TYPES[src]), idx.to(torch.int32), t.to(TYPES[src]), label.to(torch.int32)


def reference(z, idx, t, label, temperature, soft, hard, g):
    """loss, its bound, dz, its bound before the last rounding, stats, their relative bounds: 64 bits, on the CPU."""
    z, t = z.double().cpu(), t.double().cpu()
    rows, n = z.shape
    L = 150 + n // 128
    idx = idx.long().cpu()
    there = (idx >= 0) & (idx < n)
    at = torch.where(there, idx, 0)
    live = there & (t != -math.inf)
    b = torch.where(live, t / temperature, -math.inf)
    any_p = live.any(1, keepdim=True)
    most = torch.where(any_p, b.amax(1, keepdim=True), 0.0) if t.shape[1] else torch.zeros((rows, 1), dtype=torch.float64)
    b = b - most
    weight = torch.where(live, torch.exp(b), 0.0)
    total = weight.sum(1, keepdim=True)
    p = torch.where(any_p, weight / total.clamp(min=1e-300), 0.0)
    has_soft = any_p[:, 0] & (soft != 0.0)
    log_total = torch.log(total.clamp(min=1e-300))
    labelled = (label.long().cpu() >= 0) & (label.long().cpu() < n) & (hard != 0.0)
    lab = torch.where(labelled, label.long().cpu(), 0)
    largest = z.amax(1, keepdim=True)
    d = z - largest
    ea, eb = torch.exp(d / temperature), torch.exp(d)
    sa, sb = ea.sum(1, keepdim=True), eb.sum(1, keepdim=True)
    zero = torch.zeros_like(d)
    ma = (torch.where(ea > 0, ea * (d / temperature).abs(), zero)).sum(1, keepdim=True) / sa
    mb = (torch.where(eb > 0, eb * d.abs(), zero)).sum(1, keepdim=True) / sb
    q, s = ea / sa, eb / sb
    off_a, off_b = U * (L + 8 + 4 * ma), U * (L + 8 + 4 * mb)            # of the sums, relative
    size_b = torch.where(live, b.abs(), 0.0)
    off_total = U * (t.shape[1] + 30 + 4 * (p * size_b).sum(1, keepdim=True))
    off_p = U * (6 * size_b + 6 * log_total.abs() + 12) + off_total
    log_p = torch.where(live, b - log_total, 0.0)
    log_q = d.gather(1, at) / temperature - torch.log(sa)
    term = torch.where(p > 0, p * (log_p - log_q), 0.0)
    lost = torch.where(p > 0, p * (off_p * (log_p - log_q).abs() + 8 * U * (log_p.abs() + log_q.abs() + torch.log(sa) + log_total.abs())
                                   + off_a + off_total), 0.0)
    loss = torch.where(has_soft, soft * temperature ** 2 * term.sum(1), 0.0)
    bound = torch.where(has_soft, abs(soft) * temperature ** 2 * (lost.sum(1) + (t.shape[1] + 30) * U * term.abs().sum(1)), 0.0)
    log_s = d.gather(1, lab[:, None])[:, 0] - torch.log(sb[:, 0])
    loss = loss + torch.where(labelled, -hard * log_s, 0.0)
    bound = bound + torch.where(labelled, abs(hard) * (8 * U * (log_s.abs() + torch.log(sb[:, 0])) + off_b[:, 0]), 0.0) + 4 * U * loss.abs()
    g = torch.ones(rows, dtype=torch.float64) if g is None else g.double().cpu()
    teacher = torch.zeros_like(z).scatter_add_(1, at, p)
    off_teacher = torch.zeros_like(z).scatter_add_(1, at, p * (off_p + t.shape[1] * U))
    truth = torch.zeros_like(z).scatter_(1, lab[:, None], labelled.double()[:, None])
    hs, hl = has_soft.double()[:, None], labelled.double()[:, None]
    finite_a, finite_b = torch.where(ea > 0, (d / temperature).abs(), zero), torch.where(eb > 0, d.abs(), zero)
    dz = hs * soft * temperature * (q - teacher) + hl * hard * (s - truth)
    off = hs * abs(soft * temperature) * (q * (off_a + U * (4 * finite_a + 12)) + off_teacher + 4 * U * teacher)
    off = off + hl * abs(hard) * (s * (off_b + U * (4 * finite_b + 12)) + 4 * U * truth)
    # exponentials below the smallest normal number may be zero
    off = off + 2.0 ** -126 * (hs * abs(soft * temperature) + hl * abs(hard))
    return loss, bound, dz * g[:, None], (off + 4 * U * dz.abs()) * g[:, None].abs(), (largest[:, 0], sa[:, 0], sb[:, 0], off_a[:, 0], off_b[:, 0])


def check(ref, loss=None, dz=None, stats=None, has=(True, True)):
    want, bound, want_dz, bound_dz, (largest, sa, sb, off_a, off_b) = ref
    if loss is not None:
        off = (loss.double().cpu() - want).abs()
        assert (off <= bound).all(), float((off / bound.clamp(min=1e-300)).max())
    if dz is not None:
        bound_dz = bound_dz + torch.finfo(dz.dtype).eps / 2 * (want_dz.abs() + bound_dz)
        off = (dz.double().cpu() - want_dz).abs()
        assert (off <= bound_dz).all(), float((off / bound_dz.clamp(min=1e-300)).max())
    if stats is not None:
        s = stats.double().cpu()
        assert torch.equal(s[:, 0], largest)
        assert ((s[:, 1] - sa * has[0]).abs() <= off_a * sa * has[0]).all() and ((s[:, 2] - sb * has[1]).abs() <= off_b * sb * has[1]).all()


def scratch_of(rows, n):
    need = B.mv_distill_scratch_bytes(rows, n)
    return torch.full((need,), 0x77, dtype=torch.uint8, device="cuda") if need else None


SHAPES = [(1, 1, 1), (3, 2, 2), (96, 10, 4), (5, 100, 7), (6, 100, 200), (4, 1000, 50), (2, 2048, 64), (7, 2049, 3), (3, 5000, 100),
          (2, 8193, 300), (4, 16_385, 40), (2, 33_000, 20), (2, 65_537, 5), (3, 131_073, 33), (1, 300_001, 64), (1100, 300, 9), (1010, 2300, 7)]


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,n,top", SHAPES)
def test_loss_and_gradient(rows, n, top, src, dst):
    z, idx, t, label = make(rows, n, top, src, rows + n + top)
    g = torch.randn(rows, generator=torch.Generator().manual_seed(1))
    for (temperature, soft, hard), (lead, extra) in (((2.0, 0.7, 0.3), (0, 0)), ((1.0, 1.0, 0.0), (1, 3))):
        ref = reference(z, idx, t, label, temperature, soft, hard, g)
        zd, td, id_ = place(z, TYPES[src], lead, extra), place(t, TYPES[src], lead, extra), place(idx, torch.int32, lead, extra)
        loss, stats = torch.full((rows + 1,), 7.5, device="cuda"), torch.full((rows + 1, 3), 7.5, device="cuda")
        dz = torch.full((rows + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
        at = (zd, id_, td, label.cuda() if hard else None, temperature, soft, hard)
        B.mv_distill_loss(*at, loss[:rows], scratch_of(rows, n), stats=stats[:rows], dz=dz[:rows, 1:n + 1], grad=g.cuda())
        check(ref, loss[:rows], dz[:rows, 1:n + 1], stats[:rows], (True, hard != 0.0))
        dz[:rows, 1:n + 1] = 7.5
        assert (dz == 7.5).all() and (loss[rows:] == 7.5).all() and (stats[rows:] == 7.5).all()
        # the loss alone, then the gradient alone
        alone, again = torch.zeros(rows, device="cuda"), torch.zeros((rows, 3), device="cuda")
        B.mv_distill_loss(*at, alone, scratch_of(rows, n), stats=again)
        check(ref, alone, None, again, (True, hard != 0.0))
        B.mv_distill_grad(*at, again, dz[:rows, 1:n + 1], grad=g.cuda())
        check(ref, None, dz[:rows, 1:n + 1])
        dz[:rows, 1:n + 1] = 7.5
        assert (dz == 7.5).all()


@pytest.mark.parametrize("temperature,soft,hard", [(1.0, 0.5, 0.5), (0.5, 1.0, 1.0), (7.3, 2.0, 0.0), (3.0, 0.0, 1.0), (1.0, -0.5, 0.25),
                                                   (2.0, 0.0, 0.0)])
@pytest.mark.parametrize("n", [50, 3000, 140_000])
def test_weights_and_temperatures(n, temperature, soft, hard):
    z, idx, t, label = make(5, n, 12, "f32", n)
    ref = reference(z, idx, t, label, temperature, soft, hard, None)
    loss, stats, dz = torch.zeros(5, device="cuda"), torch.zeros((5, 3), device="cuda"), torch.ones((5, n), device="cuda")
    at = (z.cuda(), idx.cuda(), t.cuda(), label.cuda(), temperature, soft, hard)
    B.mv_distill_loss(*at, loss, scratch_of(5, n), stats=stats, dz=dz)
    check(ref, loss, dz, stats, (soft != 0.0, hard != 0.0))
    dz.fill_(1.0)
    B.mv_distill_grad(*at, stats, dz)
    check(ref, None, dz)
    dz.fill_(1.0)
    B.mv_distill_loss(*at, None, scratch_of(5, n), dz=dz)                # the gradient without the loss
    check(ref, None, dz)
    if soft == 0.0:                                                      # no list at all
        B.mv_distill_loss(z.cuda(), None, None, label.cuda(), temperature, 1.0, hard, loss, scratch_of(5, n), dz=dz)
        check(ref, loss, dz)


@pytest.mark.parametrize("n", [60, 3000, 140_000])
def test_masked_logits_and_empty_rows(n):
    """Coordinates that are masked by -infinity or by the lowest value, lists without an entry, rows without any term whose
    logits are NaN, lost rows beside them."""
    inf = float("inf")
    z, idx, t, label = make(9, n, 6, "f32", 5, repeats=False)
    label[:] = torch.arange(9)
    z[0, n // 2:] = -inf
    z[1, n // 2:] = torch.finfo(torch.float32).min
    idx[:2] = torch.where(idx[:2] >= n // 2, idx[:2] - n // 2, idx[:2])
    idx[0] = torch.tensor([1, 2, 3, 4, 5, 6])
    idx[2] = -1
    t[3] = -inf
    t[4, :3] = -inf
    label[2], label[3] = -1, 4
    idx[5], label[5], z[5] = -1, -1, float("nan")
    t[8, 2:] = torch.finfo(torch.float32).min
    ref = reference(z[[0, 1, 2, 3, 4, 8]], idx[[0, 1, 2, 3, 4, 8]], t[[0, 1, 2, 3, 4, 8]], label[[0, 1, 2, 3, 4, 8]], 2.0, 0.6, 0.4, None)
    z[6, 7], t[7, 0], idx[7, 0] = float("nan"), inf, 9
    loss, stats, dz = torch.ones(9, device="cuda"), torch.zeros((9, 3), device="cuda"), torch.ones((9, n), device="cuda")
    at = (z.cuda(), idx.cuda(), t.cuda(), label.cuda(), 2.0, 0.6, 0.4)
    B.mv_distill_loss(*at, loss, scratch_of(9, n), stats=stats, dz=dz)
    for again in (False, True):
        kept = [0, 1, 2, 3, 4, 8]
        check(ref, loss[kept], dz[kept])
        assert float(loss[5]) == 0.0 and (dz[5] == 0.0).all()
        assert torch.isnan(loss[6:8]).all() and torch.isnan(dz[6:8]).all()
        assert float(loss[2]) == 0.0 and (dz[2] == 0.0).all()
        assert (dz[0, n // 2:] == 0.0).all()
        dz.fill_(1.0)
        B.mv_distill_grad(*at, stats, dz)
    # the teacher lists what the student rules out
    z[0, 1] = -inf
    B.mv_distill_loss(z.cuda(), idx.cuda(), t.cuda(), None, 2.0, 0.6, 0.0, loss, scratch_of(9, n), dz=dz)
    assert float(loss[0]) == inf and torch.isfinite(dz[0]).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("n", [60, 3000, 70_000, 140_000])
def test_in_place(n, src):
    z, idx, t, label = make(7, n, 20, src, n)
    d, dz, stats = place(z, TYPES[src], 1, 3), torch.zeros((7, n), dtype=TYPES[src], device="cuda"), torch.zeros((7, 3), device="cuda")
    loss, more = torch.zeros(7, device="cuda"), torch.zeros(7, device="cuda")
    at = (idx.cuda(), t.cuda(), label.cuda(), 2.0, 0.6, 0.4)
    B.mv_distill_loss(d, *at, loss, scratch_of(7, n), stats=stats, dz=dz)
    B.mv_distill_loss(d, *at, more, scratch_of(7, n), dz=d)
    assert torch.equal(d, dz) and torch.equal(loss, more)
    d.copy_(z)
    B.mv_distill_grad(d, *at, stats, dz)
    B.mv_distill_grad(d, *at, stats, d)
    assert torch.equal(d, dz)


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(4200, 70, 5), (6200, 100, 5), (4200, 1300, 6), (4200, 2200, 6), (1100, 1500, 30), (1030, 2100, 70), (520, 20_001, 9), (300, 36_001, 5), (270, 69_700, 40)])
def test_more_rows_than_run_at_once(rows, n, top, src):
    """Rows that take turns in a workgroup, each fetched while the one before is at work; in place."""
    z, idx, t, label = make(rows, n, top, src, rows + n)
    ref = reference(z, idx, t, label, 2.0, 0.6, 0.4, None)
    loss, d, dz = torch.zeros(rows, device="cuda"), place(z, TYPES[src], 1, 3), torch.zeros((rows, n), device="cuda")
    at = (idx.cuda(), t.cuda(), label.cuda(), 2.0, 0.6, 0.4)
    B.mv_distill_loss(d, *at, loss, scratch_of(rows, n), dz=dz)
    check(ref, loss, dz)
    B.mv_distill_loss(d, *at, loss, scratch_of(rows, n), dz=d)
    assert torch.equal(d, dz.to(d.dtype))


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(3, 30, 4096), (2, 5000, 4096), (5, 1000, 1025), (2, 140_000, 3000), (2, 20_000, 4096), (260, 36_000, 4096),
                                        (50, 70_000, 4096), (3, 70_000, 2500)])
def test_long_lists(rows, n, top, src):
    z, idx, t, label = make(rows, n, top, src, top)
    ref = reference(z, idx, t, label, 2.0, 0.6, 0.4, None)
    loss, dz, stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, n), device="cuda"), torch.zeros((rows, 3), device="cuda")
    at = (z.to(TYPES[src]).cuda(), idx.cuda(), t.cuda(), label.cuda(), 2.0, 0.6, 0.4)
    B.mv_distill_loss(*at, loss, scratch_of(rows, n), stats=stats, dz=dz)
    check(ref, loss, dz)
    B.mv_distill_grad(*at, stats, dz)
    check(ref, None, dz)


def test_gradient_against_differences():
    """The loss in 64 bits on both sides of a logit: at listed coordinates, at the label, elsewhere."""
    rows, n = 3, 40
    z, idx, t, label = make(rows, n, 5, "f32", 11)
    label[:] = torch.tensor([3, 7, 1])
    dz, loss = torch.zeros((rows, n), device="cuda"), torch.zeros(rows, device="cuda")
    B.mv_distill_loss(z.cuda(), idx.cuda(), t.cuda(), label.cuda(), 1.7, 0.8, 0.3, loss, dz=dz)
    z = z.double()
    for r in range(rows):
        for v in {int(label[r]), *[int(i) for i in idx[r] if 0 <= i < n], 20, 39}:
            side = []
            for step in (1e-5, -1e-5):
                x = z.clone()
                x[r, v] += step
                side.append(float(reference(x, idx, t, label, 1.7, 0.8, 0.3, None)[0][r]))
            assert abs((side[0] - side[1]) / 2e-5 - float(dz[r, v])) <= 1e-5


def test_equal_results_each_time_and_in_a_graph():
    for rows, n in ((50, 10), (9, 5000), (3, 140_000)):
        z, idx, t, label = make(rows, n, 8, "f32", n)
        z, at = z.cuda(), (idx.cuda(), t.cuda(), label.cuda(), 2.0, 0.6, 0.4)
        loss, stats, dz, alone = (torch.zeros(s, device="cuda") for s in (rows, (rows, 3), (rows, n), (rows, n)))
        scratch = scratch_of(rows, n)

        def run(stream=None):
            B.mv_distill_loss(z, *at, loss, scratch, stats=stats, dz=dz, stream=stream)
            B.mv_distill_grad(z, *at, stats, alone, stream=stream)

        run()
        want = [x.clone() for x in (loss, stats, dz, alone)]
        for x in (loss, stats, dz, alone):
            x.zero_()
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        run(other)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((loss, stats, dz, alone), want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for _ in range(3):
            for x in (loss, stats, dz, alone):
                x.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((loss, stats, dz, alone), want))
            z.neg_()
            run()
            want = [x.clone() for x in (loss, stats, dz, alone)]


def test_many_values_beyond_32_bits():
    rows, n = 33_000, 131_072
    z = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda").normal_()
    idx = torch.randint(0, n, (rows, 4), device="cuda", dtype=torch.int32)
    t, loss = torch.randn((rows, 4), device="cuda"), torch.zeros(rows, device="cuda")
    label = torch.randint(0, n, (rows,), device="cuda", dtype=torch.int32)
    ref = reference(z[-2:], idx[-2:], t[-2:], label[-2:], 2.0, 0.6, 0.4, None)
    B.mv_distill_loss(z, idx, t, label, 2.0, 0.6, 0.4, loss, scratch_of(rows, n), dz=z)
    check(ref, loss[-2:], z[-2:])


def test_python_refusals():
    z, loss, stats = torch.zeros((4, 100), device="cuda"), torch.zeros(4, device="cuda"), torch.zeros((4, 3), device="cuda")
    idx, t, label = torch.zeros((4, 5), dtype=torch.int32, device="cuda"), torch.zeros((4, 5), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    at = (1.0, 0.5, 0.5)
    for bad in (lambda: B.mv_distill_loss(z.half(), idx, t, label, *at, loss), lambda: B.mv_distill_loss(z, idx.long(), t, label, *at, loss),
                lambda: B.mv_distill_loss(z, idx[:3], t, label, *at, loss), lambda: B.mv_distill_loss(z, idx, t[:, :4], label, *at, loss),
                lambda: B.mv_distill_loss(z, idx, t, label[:3], *at, loss), lambda: B.mv_distill_loss(z, idx, t, label.long(), *at, loss),
                lambda: B.mv_distill_loss(z, idx, t, label, *at, loss[:3]), lambda: B.mv_distill_loss(z, idx.cpu(), t, label, *at, loss),
                lambda: B.mv_distill_loss(z, idx, t, label, *at, loss, stats=stats[:2]),
                lambda: B.mv_distill_loss(z, idx, t, label, *at, loss, dz=z[:, :99]),
                lambda: B.mv_distill_loss(z, idx.t().contiguous().t(), t, label, *at, loss),
                lambda: B.mv_distill_grad(z, idx, t, label, *at, stats.double(), z)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.mv_distill_loss(z, idx, t, label, 0.0, 0.5, 0.5, loss), lambda: B.mv_distill_loss(z, idx, t, label, *at, None),
                lambda: B.mv_distill_grad(z, idx, t, label, *at, None, z)):
        with pytest.raises(B.MvError) as e:
            bad()
        assert e.value.status == B.MV_ERR_INVALID_ARG
