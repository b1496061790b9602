"""The example that runs the operators around the vote step together: a step against numpy, and that it trains."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2011_06495_amd import four_bit_training as T

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().float().cpu().numpy()


def test_a_step_follows_its_parts(oracle):
    """Norms, rows, mask, what is sent, what stays in the error buffers, and the update of a second step, from the
    gradients that the step saw and the buffers before it."""
    t = T.Trainer(workers=5, seed=3)
    t.step(0.5)
    before, err, flat = host(t.rows), host(t.err), host(t.flat)
    t.step(0.5)
    grads = [np.concatenate([host(g).ravel() for g in worker]) for worker in t.grads]
    norms, rows = host(t.norms), host(t.rows)
    assert not np.array_equal(before, rows)
    for r, g in enumerate(grads):
        norm = np.sqrt((g.astype(np.float64) ** 2).sum())
        assert abs(norms[r] - norm) <= norm * (2.0 ** -24 + 1e-9)
        c = np.float32(T.MAX_NORM) / (norms[r] + np.float32(1e-6))
        assert np.array_equal(rows[r], g * min(np.float32(1.0), c))
    ref = oracle.vote_step(rows, err, t.k)
    mask = t.mask.cpu().numpy()
    assert np.array_equal(mask.view(np.uint32), ref.mask_idx)
    sent = (rows + err)[:, mask]
    held = R.held(sent)
    left = ref.err.copy()
    left[:, mask] = (sent - held).astype(np.float32)
    assert np.array_equal(host(t.err), left)
    mean = np.zeros(t.k, np.float32)
    for row in held.astype(np.float32):
        mean += row
    mean *= np.float32(1.0) / np.float32(5)
    assert np.array_equal(host(t.mean), mean)
    want = flat.copy()
    want[mask] -= np.float32(0.5) * mean
    # torch may form the product and the difference in one rounding or in two
    assert np.allclose(host(t.flat), want, rtol=2.0 ** -23, atol=1e-9)
    t.close()


def test_it_trains():
    losses = T.train(60, workers=8)
    assert all(np.isfinite(losses))
    assert np.mean(losses[-5:]) < 0.5 * losses[0], losses
