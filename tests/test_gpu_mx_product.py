"""Products of microscaled 4-bit matrices against numpy in 64 bits.

A product of two 4-bit values is exact in fp32 and so is a power of two times it; what rounds is the sum of k products.
However they are grouped, an fp32 sum of k terms is within (k - 1) 2^-24 (1 + small) of the sum of the terms' magnitudes;
the bound below takes k 2^-23 of it, twice that, for a matrix core that cuts instead of rounding.  bf16 results are then
rounded once, 2^-8 of the result.  Where all terms are whole multiples of one power of two and the sum of their magnitudes
is below 2^24 of them, no order rounds and the result is exact."""
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
    """Codes and scales of x on the device, rows longer than they need to be, whatever lies behind the last block filled."""
    codes, scales = R.encode(x)
    words = R.pack(codes)
    c = torch.full((x.shape[0], words.shape[1] + 4), -1, dtype=torch.int32, device="cuda")
    s = torch.full((x.shape[0], (scales.shape[1] + 3) // 4 * 4 + 4), 255, dtype=torch.uint8, device="cuda")
    c[:, : words.shape[1]] = torch.from_numpy(words.view(np.int32))
    s[:, : scales.shape[1]] = torch.from_numpy(scales)
    return c, s, R.values(codes, scales, x.shape[1])


def normal(rng, rows, n):
    return (rng.standard_normal((rows, n)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)


def scratch_of(need):
    return torch.full((need,), 0x77, dtype=torch.uint8, device="cuda") if need else None


def check(got, a, b, dtype):
    """got (m x n) against a b^T."""
    k = a.shape[1]
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    bound = k * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)
    got = got.float().cpu().numpy().astype(np.float64)
    off = np.abs(got - want)
    assert (off <= bound).all(), "off by %g of the bound at %s" % (
        np.nanmax(off / np.maximum(bound, 1e-300)), np.unravel_index(np.argmax(off - bound), off.shape))


SHAPES = [(1, 1, 1), (1, 1, 32), (1, 5, 33), (2, 3, 31), (1, 1000, 2048), (3, 17, 100), (5, 64, 511), (16, 16, 128),
          (16, 100, 129), (17, 15, 512), (31, 33, 513), (8, 700, 4096), (64, 64, 64), (65, 63, 1000), (100, 130, 2000),
          (128, 128, 640), (130, 257, 544), (256, 256, 1024), (300, 200, 33), (257, 513, 1537), (12, 9, 40_000),
          (1, 3, 100_001), (33, 40, 20_000), (600, 530, 96)]


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(m, n, k, dst):
    rng = np.random.default_rng(m * 31 + n * 7 + k)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out[:m, 1:n + 1], scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    check(out[:m, 1:n + 1], a, b, TYPES[dst])
    o = out.float().cpu().numpy()
    o[:m, 1:n + 1] = 7.5
    assert (o == 7.5).all()


@pytest.mark.parametrize("m,n,k", [(1, 40, 300), (7, 33, 4096), (16, 130, 5000), (40, 50, 900), (130, 260, 2000), (300, 300, 3000)])
def test_whole_numbers_are_exact(m, n, k):
    """Values on the grid with a largest magnitude of 6, 4 or 7 in a block: scales of 1, sums of multiples of a quarter."""
    rng = np.random.default_rng(m + n + k)

    def whole(rows):
        x = rng.choice(R.GRID, size=(rows, 32 * R.blocks_of(k))) * rng.choice([-1.0, 1.0], size=(rows, 32 * R.blocks_of(k)))
        x[:, ::32] = 6.0
        return x[:, :k].astype(np.float32)

    x, y = whole(m), whole(n)
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    assert np.array_equal(a, x) and np.array_equal(b, y)
    out = torch.zeros((m, n), device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    assert np.array_equal(out.cpu().numpy().astype(np.float64), a @ b.T)


@pytest.mark.parametrize("m,n,k", [(3, 20, 200), (20, 40, 1000), (200, 300, 1100)])
def test_nan_blocks_reach_their_rows_and_columns_only(m, n, k):
    rng = np.random.default_rng(1)
    x, y = normal(rng, m, k), normal(rng, n, k)
    x[1, k - 1] = np.inf
    y[n - 1, 40] = np.nan
    a_codes, a_scales, _ = hold(x)
    b_codes, b_scales, _ = hold(y)
    out = torch.zeros((m, n), device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    lost = np.zeros((m, n), bool)
    lost[1], lost[:, n - 1] = True, True
    assert np.array_equal(np.isnan(out.cpu().numpy()), lost)


def test_scales_far_apart():
    """Blocks from 2^-127 to 2^125: products that leave fp32 upwards are infinite, downwards as fp32 has them."""
    k = 64
    x = np.zeros((4, k), np.float32)
    y = np.zeros((3, k), np.float32)
    x[0, 3], x[1, 3], x[2, 40], x[3, 40] = 3e38, 1.5 * 2.0 ** -127, 2.0, 2.0 ** 60
    y[0, 3], y[1, 3], y[2, 40] = 8.0, 2.0 ** 120, 2.0 ** -100
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    out = torch.zeros((4, 3), device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_mx_product_scratch_bytes(4, 3, k)))
    got, want = out.cpu().numpy(), a @ b.T
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32))


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 100, 2048), (2, 33, 31), (5, 130, 1000), (16, 64, 4100), (17, 70, 97),
                                   (100, 200, 513), (300, 270, 640)])
def test_linear(m, n, k, src, dst):
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    x = torch.zeros(m * (k + 3) + 1, dtype=TYPES[src], device="cuda")[1:].view(m, k + 3)[:, :k]      # unaligned rows
    x.copy_(torch.from_numpy(normal(rng, m, k)))
    w_codes, w_scales, w = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 2), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_linear(x, w_codes, w_scales, out[:m, :n], scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k)))
    check(out[:m, :n], R.held(x.float().cpu().numpy()), w, TYPES[dst])
    o = out.float().cpu().numpy()
    assert (o[m:] == 7.5).all() and (o[:, n:] == 7.5).all()


def test_linear_with_an_empty_row_and_a_lost_block():
    rng = np.random.default_rng(6)
    for m in (3, 40):
        x = normal(rng, m, 300)
        x[1] = 0.0
        x[2, 200] = np.inf
        w_codes, w_scales, w = hold(normal(rng, 50, 300))
        out = torch.full((m, 50), 7.5, device="cuda")
        B.mv_mx_linear(torch.from_numpy(x).cuda(), w_codes, w_scales, out, scratch_of(B.mv_mx_linear_scratch_bytes(m, 50, 300)))
        got = out.cpu().numpy()
        assert (got[1] == 0.0).all() and np.isnan(got[2]).all() and np.isfinite(np.delete(got, 2, 0)).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 40, 100), (5, 33, 31), (33, 17, 130), (100, 64, 200), (130, 300, 70), (700, 65, 140)])
def test_gradients_follow_their_formula(m, n, k, src):
    rng = np.random.default_rng(m + n + k)
    x = torch.from_numpy(normal(rng, m, k)).cuda().to(TYPES[src])
    dy = torch.from_numpy(normal(rng, m, n)).cuda().to(TYPES[src])
    w = normal(rng, n, k)
    wt_codes, wt_scales, wt = hold(np.ascontiguousarray(w.T))
    scratch = scratch_of(B.mv_mx_linear_grad_scratch_bytes(m, n, k))
    dx, dw = torch.zeros((m, k), dtype=TYPES[src], device="cuda"), torch.zeros((n, k), device="cuda")
    B.mv_mx_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch)
    x32, dy32 = x.float().cpu().numpy(), dy.float().cpu().numpy()
    check(dx, R.held(dy32), wt, TYPES[src])
    held_dy, held_x = R.held(np.ascontiguousarray(dy32.T)), R.held(np.ascontiguousarray(x32.T))
    check(dw, held_dy, held_x, torch.float32)
    # each alone
    dx2, dw2 = torch.zeros_like(dx), torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    B.mv_mx_linear_grad(None, dy, wt_codes, wt_scales, dx2, None, scratch)
    assert torch.equal(dx, dx2)
    B.mv_mx_linear_grad(x, dy, None, None, None, dw2, scratch)
    check(dw2, held_dy, held_x, torch.bfloat16)


def test_gradients_against_differences():
    """Where 4 bits hold x, w and dy as they are, y is linear in each: a difference of the loss sum(dy y) is the gradient's
    component, exactly (small whole numbers)."""
    rng = np.random.default_rng(21)
    m, n, k = 32, 32, 64

    def grid(rows, cols):
        x = rng.choice([-3.0, -2.0, -1.0, 0.0, 1.0, 2.0, 3.0], size=(rows, cols))
        x[::32, :] = 6.0                           # every block of rows and of columns has a scale of 1
        x[:, ::32] = 6.0
        return x.astype(np.float32)

    x, w, dy = grid(m, k), grid(n, k), grid(m, n)

    def loss(x, w):
        c, s, _ = hold(w)
        y = torch.zeros((m, n), device="cuda")
        B.mv_mx_linear(torch.from_numpy(x).cuda(), c, s, y, scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k)))
        return float((y.double().cpu() * torch.from_numpy(dy).double()).sum())

    wt_codes, wt_scales, _ = hold(np.ascontiguousarray(w.T))
    dx, dw = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    B.mv_mx_linear_grad(torch.from_numpy(x).cuda(), torch.from_numpy(dy).cuda(), wt_codes, wt_scales, dx, dw,
                        scratch_of(B.mv_mx_linear_grad_scratch_bytes(m, n, k)))
    dx, dw = dx.cpu().numpy(), dw.cpu().numpy()
    at = loss(x, w)
    for i, j in ((0, 1), (5, 7), (31, 63), (17, 33), (2, 32)):
        for what, grad in ((x, dx), (w, dw)):
            other = what.copy()
            other[i, j] = 4.0 if what[i, j] != 4.0 else 2.0
            step = float(other[i, j] - what[i, j])
            moved = loss(other, w) if what is x else loss(x, other)
            assert moved - at == step * float(grad[i, j])


def test_equal_results_each_time_and_in_a_graph():
    rng = np.random.default_rng(31)
    for m, n, k in ((1, 300, 5000), (12, 40, 30_000), (300, 200, 2000)):
        x = torch.from_numpy(normal(rng, m, k)).cuda()
        c, s, _ = hold(normal(rng, n, k))
        scratch = scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k))
        first, out = torch.zeros((m, n), device="cuda"), torch.zeros((m, n), device="cuda")
        B.mv_mx_linear(x, c, s, first, scratch)
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        B.mv_mx_linear(x, c, s, out, scratch, stream=other)
        other.synchronize()
        assert torch.equal(out, first)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.mv_mx_linear(x, c, s, out, scratch)
        for i in range(3):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)
            x.mul_(2.0)                            # powers of two: the results move with them, exactly
            first.mul_(2.0)
            B.mv_mx_linear(x, c, s, out, scratch)  # eager work between the replays
            assert torch.equal(out, first)


def test_python_refusals():
    rng = np.random.default_rng(1)
    c, s, _ = hold(normal(rng, 10, 100))
    x, y = torch.zeros((4, 100), device="cuda"), torch.zeros((4, 10), device="cuda")
    scratch = scratch_of(B.mv_mx_linear_scratch_bytes(4, 10, 100))
    for bad in (lambda: B.mv_mx_linear(x.double(), c, s, y, scratch), lambda: B.mv_mx_linear(x, c[:9], s, y, scratch),
                lambda: B.mv_mx_linear(x[:3], c, s, y, scratch), lambda: B.mv_mx_linear(x, c, s, y.t(), scratch),
                lambda: B.mv_mx_linear(x, c[:, :12], s, y, scratch), lambda: B.mv_mx_linear(x, c, s, y, scratch.cpu()),
                lambda: B.mv_mx_product(c, s, c, s, 200, torch.zeros((10, 10), device="cuda"), scratch),
                lambda: B.mv_mx_linear_grad(x, y.bfloat16(), c, s, None, torch.zeros((10, 100), device="cuda"), scratch)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.MvError) as e:
        B.mv_mx_linear(x, c, s, y, scratch[:1])
    assert e.value.status == B.MV_ERR_INVALID_ARG


@pytest.mark.parametrize("m,n,k", [(3, 5, 9_000_001), (20, 18, 2_000_033)])
def test_long_sums_of_few_rows(m, n, k):
    """The products of workers' whole gradients with each other: k is the long side, split over the units."""
    rng = np.random.default_rng(k)
    base = rng.standard_normal(4099).astype(np.float32)
    x, y = (np.stack([np.roll(np.resize(base, k), 7 * r + s) for r in range(rows)]) for rows, s in ((m, 0), (n, 3)))
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    out = torch.zeros((m, n), device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    check(out, a, b, torch.float32)


@pytest.mark.parametrize("words,places", [((1 << 20) + 4, 64), ((1 << 22) + 4, 64), (64, (1 << 22) + 4)])
def test_rows_far_apart(words, places):
    """Rows of codes 4 and 16 MB apart, and rows of scales 4 MB: offsets inside a tile near and beyond 32 bits."""
    m, n, k = 40, 20, 300
    rng = np.random.default_rng(words)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    far = torch.zeros((m, words), dtype=torch.int32, device="cuda")
    far_scales = torch.zeros((m, places), dtype=torch.uint8, device="cuda")
    far[:, :40] = a_codes[:, :40]
    far_scales[:, :12] = a_scales[:, :12]
    for first in (True, False):
        out = torch.zeros((m, n) if first else (n, m), device="cuda")
        sides = (far, far_scales, b_codes, b_scales) if first else (b_codes, b_scales, far, far_scales)
        B.mv_mx_product(*sides, k, out, scratch_of(B.mv_mx_product_scratch_bytes(*out.shape, k)))
        check(out, a, b, torch.float32) if first else check(out, b, a, torch.float32)


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2100, 2070, 20), (2049, 2100, 257), (1030, 4500, 768), (2500, 2100, 1000), (2100, 2200, 1056),
                                   (3600, 3500, 1100)])
def test_many_tiles(m, n, k, dst):
    """More tiles than units, with few steps along k and with more of them, and the large tiles."""
    rng = np.random.default_rng(m + n + k)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_mx_product(a_codes, a_scales, b_codes, b_scales, k, out[:m, 1:n + 1], scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    check(out[:m, 1:n + 1], a, b, TYPES[dst])
    o = out.float().cpu().numpy()
    o[:m, 1:n + 1] = 7.5
    assert (o == 7.5).all()


@pytest.mark.parametrize("m,n,k", [(1000, 130, 4500), (300, 900, 5000), (2000, 1100, 1300)])
def test_gradients_of_many_tiles(m, n, k):
    rng = np.random.default_rng(m + n + k)
    x, dy = torch.from_numpy(normal(rng, m, k)).cuda().bfloat16(), torch.from_numpy(normal(rng, m, n)).cuda().bfloat16()
    wt_codes, wt_scales, wt = hold(normal(rng, k, n))
    dx, dw = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    B.mv_mx_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch_of(B.mv_mx_linear_grad_scratch_bytes(m, n, k)))
    x32, dy32 = x.float().cpu().numpy(), dy.float().cpu().numpy()
    check(dx, R.held(dy32), wt, torch.float32)
    check(dw, R.held(np.ascontiguousarray(dy32.T)), R.held(np.ascontiguousarray(x32.T)), torch.float32)


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 600, 9000), (2, 530, 13_001), (16, 513, 17_000), (5, 12_300, 2100), (1, 12_500, 4500),
                                   (12, 4200, 4100), (16, 9000, 4100), (40, 5000, 2500)])
def test_few_rows_of_values(m, n, k, src):
    """Several turns of a wavefront, 32 of the many rows, and on both sides of what workgroups quantise for themselves."""
    rng = np.random.default_rng(m + n + k)
    x = torch.from_numpy(normal(rng, m, k)).cuda().to(TYPES[src])
    w_codes, w_scales, w = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 2), 7.5, device="cuda")
    B.mv_mx_linear(x, w_codes, w_scales, out[:m, :n], scratch_of(B.mv_mx_linear_scratch_bytes(m, n, k)))
    check(out[:m, :n], R.held(x.float().cpu().numpy()), w, torch.float32)
    assert (out[m:] == 7.5).all() and (out[:, n:] == 7.5).all()
    codes, scales = torch.zeros_like(w_codes[:1]).expand(m, -1).contiguous(), torch.zeros_like(w_scales[:1]).expand(m, -1).contiguous()
    B.mv_mx_encode(x, codes, scales)
    again = torch.zeros((m, n), device="cuda")
    B.mv_mx_product(codes, scales, w_codes, w_scales, k, again, scratch_of(B.mv_mx_product_scratch_bytes(m, n, k)))
    check(again, R.held(x.float().cpu().numpy()), w, torch.float32)
