"""Products of 8-bit matrices with a scale for each block of 128 against numpy in 64 bits.

A product of two 8-bit values has eight bits and so is exact in fp32, and so is a power of two times it; what rounds is the sum of
k products.  However they are grouped, an fp32 sum of k terms is within (k - 1) 2^-24 (1 + small) of the sum of the terms'
magnitudes; the bound below takes k 2^-23 of it, twice that, for a matrix core that cuts instead of rounding.  bf16 results
may come from instructions that cut seven of eight products at 2^-13 of the largest, 7 2^-13 of the magnitudes' sum, and are then
rounded once, 2^-8 of the result.  Where all terms are whole multiples of one power of two and the sum of their
magnitudes is below 2^24 of them, no order rounds and the result is exact."""
import numpy as np
import pytest
import torch

import f8_reference as R
from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def hold(x):
    """Codes and scales of x on the device, rows longer than they need to be, whatever lies behind the last block filled."""
    codes, scales = R.encode(x)
    c = torch.full((x.shape[0], codes.shape[1] + 16), -1, dtype=torch.int8, device="cuda").view(torch.uint8)
    s = torch.full((x.shape[0], (scales.shape[1] + 3) // 4 * 4 + 4), 255, dtype=torch.uint8, device="cuda")
    c[:, : codes.shape[1]] = torch.from_numpy(codes)
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
    bound = k * 2.0 ** -23 * size
    if dtype == torch.bfloat16:
        bound += 7 * 2.0 ** -13 * size
        bound += 2.0 ** -8 * (np.abs(want) + bound)
    got = got.float().cpu().numpy().astype(np.float64)
    off = np.abs(got - want)
    assert (off <= bound).all(), "off by %g of the bound at %s" % (
        np.nanmax(off / np.maximum(bound, 1e-300)), np.unravel_index(np.argmax(off - bound), off.shape))


SHAPES = [(1, 1, 1), (1, 1, 128), (1, 5, 129), (2, 3, 127), (1, 1000, 2048), (3, 17, 100), (5, 64, 511), (16, 16, 512),
          (16, 100, 513), (17, 15, 2048), (31, 33, 2049), (8, 700, 4096), (64, 64, 64), (65, 63, 1000), (100, 130, 2000),
          (128, 128, 640), (130, 257, 544), (256, 256, 1024), (300, 200, 33), (257, 513, 1537), (12, 9, 40_000),
          (1, 3, 100_001), (33, 40, 20_000), (600, 530, 96)]


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(m, n, k, dst):
    rng = np.random.default_rng(m * 31 + n * 7 + k)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out[:m, 1:n + 1], scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    check(out[:m, 1:n + 1], a, b, TYPES[dst])
    o = out.float().cpu().numpy()
    o[:m, 1:n + 1] = 7.5
    assert (o == 7.5).all()


@pytest.mark.parametrize("m,n,k", [(1, 40, 300), (7, 33, 4096), (16, 130, 5000), (40, 50, 900), (130, 260, 2000), (300, 300, 3000),
                                   (20, 18, 200_000), (2100, 2200, 300), (3600, 3500, 200), (1024, 2048, 5632), (260, 390, 1536),
                                   (150, 700, 2560)])
def test_whole_numbers_are_exact(m, n, k):
    """Whole numbers up to 15, which any block with a largest magnitude up to 15 holds; a result's products come to less than
    2^24: half of a long row are zeros, and the others mostly small."""
    rng = np.random.default_rng(m + n + k)
    most = 15 if k <= 5000 else 3

    def whole(rows):
        x = rng.integers(-most, most + 1, size=(rows, k)).astype(np.float32)
        x[rng.random((rows, k)) < 0.5] = 0.0
        return x

    x, y = whole(m), whole(n)
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    assert np.array_equal(a, x) and np.array_equal(b, y)
    assert float((np.abs(x) @ np.abs(y).T).max()) < 2.0 ** 24
    want = torch.from_numpy(x @ y.T)
    for dst in TYPES.values():                          # of eight products the largest is below 2^8 times the smallest
        out = torch.zeros((m, n), dtype=dst, device="cuda")
        B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
        assert torch.equal(out.cpu(), want.to(dst))


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 20, 200), (20, 40, 1000), (200, 300, 1100), (2100, 2200, 200), (2100, 4400, 700)])
def test_nan_blocks_reach_their_rows_and_columns_only(m, n, k, dst):
    rng = np.random.default_rng(1)
    x, y = normal(rng, m, k), normal(rng, n, k)
    x[1, k - 1] = np.inf
    y[n - 1, 40] = np.nan
    a_codes, a_scales, _ = hold(x)
    b_codes, b_scales, _ = hold(y)
    out = torch.zeros((m, n), dtype=TYPES[dst], device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    lost = np.zeros((m, n), bool)
    lost[1], lost[:, n - 1] = True, True
    assert np.array_equal(torch.isnan(out).cpu().numpy(), lost)


def test_scales_far_apart():
    """Blocks from 2^-127 to 2^120: products that leave fp32 upwards are infinite, downwards as fp32 has them."""
    k = 200
    x = np.zeros((4, k), np.float32)
    y = np.zeros((3, k), np.float32)
    x[0, 3], x[1, 3], x[2, 140], x[3, 140] = 3e38, 1.5 * 2.0 ** -127, 2.0, 2.0 ** 60
    y[0, 3], y[1, 3], y[2, 140] = 8.0, 2.0 ** 120, 2.0 ** -100
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    out = torch.zeros((4, 3), device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(4, 3, k)))
    got, want = out.cpu().numpy(), a @ b.T
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32))


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 100, 2048), (2, 33, 31), (5, 130, 1000), (16, 64, 4100), (17, 70, 97),
                                   (40, 300, 1300), (100, 200, 513), (300, 270, 640)])
def test_linear(m, n, k, src, dst):
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    x = torch.zeros(m * (k + 3) + 1, dtype=TYPES[src], device="cuda")[1:].view(m, k + 3)[:, :k]      # unaligned rows
    x.copy_(torch.from_numpy(normal(rng, m, k)))
    w_codes, w_scales, w = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 2), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_f8_linear(x, w_codes, w_scales, out[:m, :n], scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k)))
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
        B.mv_f8_linear(torch.from_numpy(x).cuda(), w_codes, w_scales, out, scratch_of(B.mv_f8_linear_scratch_bytes(m, 50, 300)))
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
    scratch = scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k))
    dx, dw = torch.zeros((m, k), dtype=TYPES[src], device="cuda"), torch.zeros((n, k), device="cuda")
    B.mv_f8_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch)
    x32, dy32 = x.float().cpu().numpy(), dy.float().cpu().numpy()
    check(dx, R.held(dy32), wt, TYPES[src])
    held_dy, held_x = R.held(np.ascontiguousarray(dy32.T)), R.held(np.ascontiguousarray(x32.T))
    check(dw, held_dy, held_x, torch.float32)
    # each alone
    dx2, dw2 = torch.zeros_like(dx), torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    B.mv_f8_linear_grad(None, dy, wt_codes, wt_scales, dx2, None, scratch)
    check(dx2, R.held(dy32), wt, TYPES[src])             # alone, its sums may be another kernel's, in another order
    B.mv_f8_linear_grad(x, dy, None, None, None, dw2, scratch)
    check(dw2, held_dy, held_x, torch.bfloat16)


def test_gradients_against_differences():
    """Where 8 bits hold x, w and dy as they are, y is linear in each: a difference of the loss sum(dy y) is the gradient's
    component, exactly (small whole numbers)."""
    rng = np.random.default_rng(21)
    m, n, k = 32, 32, 200

    def grid(rows, cols):
        return rng.integers(-7, 8, size=(rows, cols)).astype(np.float32)

    x, w, dy = grid(m, k), grid(n, k), grid(m, n)

    def loss(x, w):
        c, s, _ = hold(w)
        y = torch.zeros((m, n), device="cuda")
        B.mv_f8_linear(torch.from_numpy(x).cuda(), c, s, y, scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k)))
        return float((y.double().cpu() * torch.from_numpy(dy).double()).sum())

    wt_codes, wt_scales, _ = hold(np.ascontiguousarray(w.T))
    dx, dw = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    B.mv_f8_linear_grad(torch.from_numpy(x).cuda(), torch.from_numpy(dy).cuda(), wt_codes, wt_scales, dx, dw,
                        scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k)))
    dx, dw = dx.cpu().numpy(), dw.cpu().numpy()
    at = loss(x, w)
    for i, j in ((0, 1), (5, 7), (31, 199), (17, 128), (2, 32)):
        for what, grad in ((x, dx), (w, dw)):
            other = what.copy()
            other[i, j] = 9.0
            step = float(other[i, j] - what[i, j])
            moved = loss(other, w) if what is x else loss(x, other)
            assert moved - at == step * float(grad[i, j])


def test_equal_results_each_time_and_in_a_graph():
    rng = np.random.default_rng(31)
    for m, n, k in ((1, 300, 5000), (12, 40, 30_000), (300, 200, 2000)):
        x = torch.from_numpy(normal(rng, m, k)).cuda()
        c, s, _ = hold(normal(rng, n, k))
        scratch = scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k))
        first, out = torch.zeros((m, n), device="cuda"), torch.zeros((m, n), device="cuda")
        B.mv_f8_linear(x, c, s, first, scratch)
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        B.mv_f8_linear(x, c, s, out, scratch, stream=other)
        other.synchronize()
        assert torch.equal(out, first)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.mv_f8_linear(x, c, s, out, scratch)
        for i in range(3):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)
            x.mul_(2.0)                            # powers of two: the results move with them, exactly
            first.mul_(2.0)
            B.mv_f8_linear(x, c, s, out, scratch)  # eager work between the replays
            assert torch.equal(out, first)


def test_python_refusals():
    rng = np.random.default_rng(1)
    c, s, _ = hold(normal(rng, 10, 100))
    x, y = torch.zeros((4, 100), device="cuda"), torch.zeros((4, 10), device="cuda")
    scratch = scratch_of(B.mv_f8_linear_scratch_bytes(4, 10, 100))
    for bad in (lambda: B.mv_f8_linear(x.double(), c, s, y, scratch), lambda: B.mv_f8_linear(x, c[:9], s, y, scratch),
                lambda: B.mv_f8_linear(x[:3], c, s, y, scratch), lambda: B.mv_f8_linear(x, c, s, y.t(), scratch),
                lambda: B.mv_f8_linear(x, c[:, :112], s, y, scratch), lambda: B.mv_f8_linear(x, c, s, y, scratch.cpu()),
                lambda: B.mv_f8_product(c, s, c, s, 200, torch.zeros((10, 10), device="cuda"), scratch),
                lambda: B.mv_f8_linear_grad(x, y.bfloat16(), c, s, None, torch.zeros((10, 100), device="cuda"), scratch)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.MvError) as e:
        B.mv_f8_linear(x, c, s, y, scratch[:1])
    assert e.value.status == B.MV_ERR_INVALID_ARG


@pytest.mark.parametrize("m,n,k", [(3, 5, 3_000_001), (20, 18, 1_000_033)])
def test_long_sums_of_few_rows(m, n, k):
    """The products of workers' whole gradients with each other: k is the long side, split over the units."""
    rng = np.random.default_rng(k)
    base = rng.standard_normal(4099).astype(np.float32)
    x, y = (np.stack([np.roll(np.resize(base, k), 7 * r + s) for r in range(rows)]) for rows, s in ((m, 0), (n, 3)))
    a_codes, a_scales, a = hold(x)
    b_codes, b_scales, b = hold(y)
    out = torch.zeros((m, n), device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    check(out, a, b, torch.float32)


@pytest.mark.parametrize("length,places", [((1 << 22) + 16, 64), ((1 << 24) + 16, 64), (512, (1 << 22) + 4)])
def test_rows_far_apart(length, places):
    """Rows of codes 4 and 16 MB apart, and rows of scales 4 MB: offsets inside a tile near and beyond 32 bits."""
    m, n, k = 40, 20, 300
    rng = np.random.default_rng(length)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    far = torch.zeros((m, length), dtype=torch.uint8, device="cuda")
    far_scales = torch.zeros((m, places), dtype=torch.uint8, device="cuda")
    far[:, :384] = a_codes[:, :384]
    far_scales[:, :4] = a_scales[:, :4]
    for first in (True, False):
        out = torch.zeros((m, n) if first else (n, m), device="cuda")
        sides = (far, far_scales, b_codes, b_scales) if first else (b_codes, b_scales, far, far_scales)
        B.mv_f8_product(*sides, k, out, scratch_of(B.mv_f8_product_scratch_bytes(*out.shape, k)))
        check(out, a, b, torch.float32) if first else check(out, b, a, torch.float32)


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2100, 2070, 20), (2049, 2100, 257), (1030, 4500, 768), (2500, 2100, 1000), (2100, 2200, 1056),
                                   (3600, 3500, 1100), (2100, 2200, 500), (3500, 3520, 300),
                                   (3500, 3520, 130), (4300, 2100, 650)])
def test_many_tiles(m, n, k, dst):
    """More tiles than units, with few steps along k and with more of them, and the large tiles."""
    rng = np.random.default_rng(m + n + k)
    a_codes, a_scales, a = hold(normal(rng, m, k))
    b_codes, b_scales, b = hold(normal(rng, n, k))
    out = torch.full((m + 1, n + 3), 7.5, dtype=TYPES[dst], device="cuda")
    B.mv_f8_product(a_codes, a_scales, b_codes, b_scales, k, out[:m, 1:n + 1], scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
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
    B.mv_f8_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch_of(B.mv_f8_linear_grad_scratch_bytes(m, n, k)))
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
    B.mv_f8_linear(x, w_codes, w_scales, out[:m, :n], scratch_of(B.mv_f8_linear_scratch_bytes(m, n, k)))
    check(out[:m, :n], R.held(x.float().cpu().numpy()), w, torch.float32)
    assert (out[m:] == 7.5).all() and (out[:, n:] == 7.5).all()
    codes, scales = torch.zeros_like(w_codes[:1]).expand(m, -1).contiguous(), torch.zeros_like(w_scales[:1]).expand(m, -1).contiguous()
    B.mv_f8_encode(x, codes, scales)
    again = torch.zeros((m, n), device="cuda")
    B.mv_f8_product(codes, scales, w_codes, w_scales, k, again, scratch_of(B.mv_f8_product_scratch_bytes(m, n, k)))
    check(again, R.held(x.float().cpu().numpy()), w, torch.float32)
