"""Products of microscaled 4-bit matrices whose results are exact.  All values lie on the 4-bit grid at their block's scale,
so quantising changes nothing, every product is a multiple of a quarter, and as long as the magnitudes of a result's
products add up to less than 2^22, 2^24 quarters, no order of adding them up in fp32 rounds: a result is right or wrong.

Long sums are split over workgroups and joined, with more than 16 splits by groups of threads; up to 16 rows of codes and 64
rows of values have a kernel of their own, which holds them in up to 144 KB of LDS."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def hold(x):
    codes, scales = R.encode(x)
    words = R.pack(codes)
    c = torch.full((x.shape[0], words.shape[1] + 4), -1, dtype=torch.int32, device="cuda")
    s = torch.full((x.shape[0], (scales.shape[1] + 3) // 4 * 4 + 4), 255, dtype=torch.uint8, device="cuda")
    c[:, : words.shape[1]] = torch.from_numpy(words.view(np.int32))
    s[:, : scales.shape[1]] = torch.from_numpy(scales)
    return c, s


def dense(rng, rows, k):
    """Values of the whole grid; each block has a 6, so its scale is 1."""
    x = rng.choice(R.GRID, size=(rows, k)) * rng.choice([-1.0, 1.0], size=(rows, k))
    x[:, ::32] = rng.choice([-6.0, 6.0], size=x[:, ::32].shape)
    return x.astype(np.float32)


def thin(rng, rows, k):
    """Halves, ones and zeros: of 9 million of each a result's products come to 1.7 million."""
    return rng.choice(np.array([0.0, 0.0, 0.0, 0.5, -0.5, 1.0, -1.0], np.float32), size=(rows, k))


def scratch_of(need):
    return torch.full((need,), 0x77, dtype=torch.uint8, device="cuda") if need else None


def exact(x, y):
    assert (np.abs(x).astype(np.float64) @ np.abs(y).astype(np.float64).T).max() < 2.0 ** 22
    return x.astype(np.float64) @ y.astype(np.float64).T


def same(out, m, n, want):
    """out's m x n values at column 1 are want, and nothing around them was written."""
    got = out.float().cpu().numpy()
    assert np.array_equal(got[:m, 1:n + 1], torch.from_numpy(want).to(out.dtype).float().numpy())
    got[:m, 1:n + 1] = 7.5
    assert (got == 7.5).all()


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(12, 9, 40_000), (1, 3, 100_001), (20, 18, 300_007), (130, 40, 30_000), (20, 18, 2_000_033),
                                   (3, 5, 9_000_001), (2, 1, 4_194_305)])
def test_long_sums(m, n, k, dst):
    rng = np.random.default_rng(k)
    make = dense if k < 400_000 else thin
    x, y = make(rng, m, k), make(rng, n, k)
    if make is thin:                                  # the last, ragged block and the ends of the runs count in every result
        x[:, [0, k // 2, k - 1]] = y[:, [0, k // 2, k - 1]] = 1.0
    a, b = hold(x), hold(y)
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_product(*a, *b, k, out[:m, 1:n + 1], scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    same(out, m, n, exact(x, y))


@pytest.mark.parametrize("where", ["first", "last", "ragged"])
@pytest.mark.parametrize("m,n,k", [(3, 5, 9_000_001), (20, 18, 2_000_033), (12, 9, 40_009)])
def test_one_value_of_a_long_sum(m, n, k, where):
    """All that a result has is one value: in the first block, the last whole one or the ragged one behind it."""
    at = {"first": 17, "last": k // 32 * 32 - 1, "ragged": k - 1}[where]
    x, y = np.zeros((m, k), np.float32), np.zeros((n, k), np.float32)
    x[:, at], y[:, at] = np.arange(1, m + 1) % 4, 1.0 + np.arange(n) % 3
    out = torch.full((m + 1, n + 3), 7.5, device="cuda")
    B.mv_mx_product(*hold(x), *hold(y), k, out[:m, 1:n + 1], scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    same(out, m, n, exact(x, y))


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(16, 600, 15_000), (16, 513, 8192), (9, 700, 20_001), (16, 12_400, 8190), (600, 16, 14_337),
                                   (3, 520, 65_000)])
def test_few_rows_of_codes_in_much_lds(m, n, k, dst):
    """The kernel for few rows with 74 to 143 KB of LDS, one and two tiles of the many rows, the few ones on either side."""
    rng = np.random.default_rng(m + n + k)
    x, y = dense(rng, m, k), dense(rng, n, k)
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_product(*hold(x), *hold(y), k, out[:m, 1:n + 1], scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    same(out, m, n, exact(x, y))


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,n,k", [(17, 300, 1500), (20, 1000, 700), (31, 4090, 601), (32, 33, 2000), (33, 500, 1999), (40, 1000, 1000),
                                   (48, 77, 640), (63, 2000, 601), (64, 1001, 1990), (64, 16, 2050), (16, 520, 8192), (16, 515, 8161)])
def test_linear_of_few_rows(m, n, k, src, dst):
    """Every workgroup quantises up to 64 rows of values for itself: two and four tiles of them, several turns of 512 values,
    ragged ends, up to 79 KB of LDS."""
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    values, weights = dense(rng, m, k), dense(rng, n, k)
    x = torch.zeros(m * (k + 3) + 1, dtype=TYPES[src], device="cuda")[1:].view(m, k + 3)[:, :k]      # unaligned rows
    x.copy_(torch.from_numpy(values))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_linear(x, *hold(weights), out[:m, 1:n + 1], scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k)))
    same(out, m, n, exact(values, weights))


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(20, 100, 1300), (40, 50, 300), (64, 200, 1111)])
def test_linear_of_few_rows_rounds_as_the_definition(m, n, k, src):
    """Values that 4 bits do not hold, one row of zeros and one lost block: an fp32 sum of k terms is off by less than k 2^-23 of
    the sum of their magnitudes, whatever their order."""
    rng = np.random.default_rng(m + n + k)
    x = (rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))).astype(np.float32)
    x[1] = 0.0
    x[m - 1, k - 2] = np.inf
    x = torch.from_numpy(x).to(TYPES[src])
    w = rng.standard_normal((n, k)).astype(np.float32)
    out = torch.full((m, n), 7.5, device="cuda")
    B.mv_mx_linear(x.cuda(), *hold(w), out, scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k)))
    got = out.cpu().numpy().astype(np.float64)
    a, b = R.held(x[:m - 1].float().numpy()), R.held(w)
    assert (got[1] == 0.0).all() and np.isnan(got[m - 1]).all()
    assert (np.abs(got[:m - 1] - a @ b.T) <= k * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()


@pytest.mark.parametrize("m,n,k", [(64, 300, 20), (4, 40, 700), (5000, 20, 18), (3000, 140, 500), (300, 600, 5000), (2300, 1100, 900)])
def test_gradients(m, n, k):
    """Both gradients of a layer, one launch for both, the sums over m split where m is long and over n where n is."""
    rng = np.random.default_rng(m + n + k)

    def whole(rows, cols):
        v = dense(rng, rows, cols)
        v[::32, :] = 6.0                              # in every block of a column, too, the scale is 1
        return v

    x, dy, wt = whole(m, k), whole(m, n), dense(rng, k, n)
    dx, dw = (torch.full((rows + 1, k + 3), 7.5, device="cuda") for rows in (m, n))
    B.mv_mx_linear_grad(torch.from_numpy(x).cuda(), torch.from_numpy(dy).cuda(), *hold(wt), dx[:m, 1:k + 1], dw[:n, 1:k + 1],
                        scratch_of(B.mv_mx_linear_grad_scratch_bytes(m, n, k)))
    same(dx, m, k, exact(dy, wt))
    same(dw, n, k, exact(np.ascontiguousarray(dy.T), np.ascontiguousarray(x.T)))
