"""Layer norm, 8-bit products and distillation together, as the example's options run them: a worker's pass stage by stage
against 64 bits, each from what the stage before left, and the gradients that the vote step then sees.

With u = 2^-24: sums of k products are within k 2^-23 of the sum of their magnitudes (here both factors are what 8 bits hold,
and results are fp32); the layer norm's and the distillation's own bounds stand in their tests, and are taken here with
room: 200 u of the sum of the magnitudes of what a result is made of."""
import numpy as np
import pytest
import torch

import f8_reference as R
from paper_2011_06495_amd import binding as B
from paper_2011_06495_amd import four_bit_training as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def near(got, want, size):
    assert (np.abs(host(got) - want) <= size).all(), float((np.abs(host(got) - want) / np.maximum(size, 1e-300)).max())


def held(x):
    return R.held(np.ascontiguousarray(x).astype(np.float32))


def check_product(got, a, b):
    """a b^T of what 8 bits hold of both."""
    a, b = held(a), held(b)
    near(got, a @ b.T, a.shape[1] * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T))


def test_a_pass_stage_by_stage(monkeypatch):
    t = T.Trainer(workers=3, seed=5, eight_bit=True, norm=True, teacher=4)
    for w, p in zip(t.weights, t.params):
        w.hold(p)
    t.norm[0].copy_(1.0 + 0.1 * torch.randn(T.HIDDEN, generator=t.gen, device="cuda"))
    t.norm[1].copy_(0.1 * torch.randn(T.HIDDEN, generator=t.gen, device="cuda"))
    x, y = t.batch()
    seen = {}

    def watched(name):
        call = getattr(B, name)

        def run(*args, **kw):
            before = [a.clone() if isinstance(a, torch.Tensor) and a.dtype != torch.uint8 else a for a in args]
            call(*args, **kw)
            seen.setdefault(name, []).append((before, [a.clone() if isinstance(a, torch.Tensor) else a for a in args], kw))

        return run

    for name in ("mv_layernorm_forward", "mv_layernorm_backward", "mv_distill_loss"):
        monkeypatch.setattr(B, name, watched(name))
    for name in ("linear", "linear_grad"):
        monkeypatch.setattr(T.EightBitWeights, name, staticmethod(watched("mv_f8_" + name)))
    loss = t.gradients(x, y, t.grads[0])
    w1, w2 = host(t.params[0]), host(t.params[1])

    (first, first_after, _), (_, second_after, _) = seen["mv_f8_linear"]
    check_product(first_after[3], host(x), w1)
    h = np.maximum(host(first_after[3]), 0.0)
    _, after, _ = seen["mv_layernorm_forward"][0]
    assert np.array_equal(host(after[0]), h)
    gamma, beta = host(t.norm[0]), host(t.norm[1])
    mean = h.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + T.EPS)
    hat = (h - mean) * rstd
    near(after[4], hat * gamma + beta, 200 * U * ((np.abs(hat) + 1) * np.abs(gamma) + np.abs(beta)))
    h2 = host(after[4])
    check_product(second_after[3], h2, w2)
    z = host(second_after[3])

    _, after, kw = seen["mv_distill_loss"][0]
    idx, top, labels = (a.cpu().numpy() for a in after[1:4])
    assert np.array_equal(labels, y.cpu().numpy()) and all(len(set(r)) == 4 for r in idx)
    p = np.exp(top / T.TEMPERATURE - top.max(1, keepdims=True) / T.TEMPERATURE)
    p /= p.sum(1, keepdims=True)
    log_q = z / T.TEMPERATURE - np.log(np.exp(z / T.TEMPERATURE).sum(1, keepdims=True))
    log_s = z - np.log(np.exp(z).sum(1, keepdims=True))
    rows = np.arange(T.BATCH)
    terms = p * (np.log(p) - np.take_along_axis(log_q, idx, 1))
    want = 0.5 * T.TEMPERATURE ** 2 * terms.sum(1) - 0.5 * log_s[rows, labels]
    near(after[7], want, 200 * U * (np.abs(log_q).max(1) + np.abs(log_s).max(1) + np.abs(z).max(1) + 1) * 4)
    assert abs(float(loss) - want.mean()) <= 1e-5 * (1 + abs(want.mean()))
    teacher = np.zeros_like(z)
    np.put_along_axis(teacher, idx, p, 1)
    truth = np.eye(T.CLASSES)[labels]
    dz = (0.5 * T.TEMPERATURE * (np.exp(log_q) - teacher) + 0.5 * (np.exp(log_s) - truth)) / T.BATCH
    near(kw["dz"], dz, 200 * U * (np.abs(z).max() + 1) * 2.0 / T.BATCH)
    dz = host(kw["dz"])

    (_, second_after, _), (before, _, _) = seen["mv_f8_linear_grad"]
    check_product(second_after[4], dz, w2.T)
    check_product(t.grads[0][1], dz.T, h2.T)
    dh2 = host(second_after[4])
    mean, rstd = host(t.h_mean)[:, None], host(t.h_rstd)[:, None]
    hat, d = (h - mean) * rstd, dh2 * gamma
    dh = rstd * (d - d.mean(1, keepdims=True) - hat * (d * hat).mean(1, keepdims=True))
    dh_seen = seen["mv_layernorm_backward"][0][1][5]
    near(dh_seen, dh, 200 * U * rstd * (np.abs(d) + np.abs(d).mean(1, keepdims=True) + np.abs(hat) * np.abs(d * hat).mean(1, keepdims=True)))
    near(t.grads[0][2], (dh2 * hat).sum(0), 200 * U * np.abs(dh2 * hat).sum(0))
    near(t.grads[0][3], dh2.sum(0), 200 * U * np.abs(dh2).sum(0))
    dh = host(dh_seen) * (h > 0)
    assert np.array_equal(host(before[1]), dh)
    check_product(t.grads[0][0], dh.T, host(x).T)
    t.close()


@pytest.mark.parametrize("options", [dict(eight_bit=True), dict(norm=True), dict(teacher=3), dict(eight_bit=True, norm=True, teacher=10)])
def test_it_runs(options):
    t = T.Trainer(workers=4, seed=1, **options)
    before = t.flat.clone()
    for _ in range(3):
        assert torch.isfinite(t.step(0.5))
    assert all(torch.isfinite(g).all() and (g != 0.0).any() for worker in t.grads for g in worker)
    assert len(t.sizes) == (4 if "norm" in options else 2) and t.d == t.flat.numel()
    assert torch.isfinite(t.flat).all() and not torch.equal(t.flat, before)
    # what went into the rows is what the passes left, clipped
    rows = torch.stack([torch.cat([g.reshape(-1) for g in worker]) for worker in t.grads])
    assert torch.equal(t.rows, rows * t.coefs[:, None])
    t.close()


def test_a_pass_in_a_graph():
    """A worker's pass captured, and replayed with eager passes in between on the same buffers."""
    t = T.Trainer(workers=2, seed=2, eight_bit=True, norm=True, teacher=4)
    for w, p in zip(t.weights, t.params):
        w.hold(p)
    x, y = t.batch()
    t.gradients(x, y, t.grads[0])
    want = [g.clone() for g in t.grads[0]]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        t.gradients(x, y, t.grads[0])
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.gradients(x, y, t.grads[0])
    for _ in range(3):
        for a in t.grads[0]:
            a.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(t.grads[0], want))
        t.gradients(x, y, t.grads[1])
        assert all(torch.equal(a, b) for a, b in zip(t.grads[1], want))
    t.close()
