"""8-bit floating point by blocks of 128: quantising rows and columns and reading back, against numpy in 64 bits, byte by byte."""
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


def place(x, dtype, lead, extra):
    """x on the device, its rows `extra` values apart and `lead` values into its memory."""
    rows, n = x.shape
    flat = torch.full((lead + rows * (n + extra),), 3.0, dtype=dtype, device="cuda")
    out = flat[lead:].view(rows, n + extra)[:, :n]
    out.copy_(torch.from_numpy(x))
    return out


def room(rows, n, more=0):
    """Codes and scales with a row more than needed and longer rows, all filled."""
    return (torch.full((rows + 1, B.mv_f8_row_bytes(n) + 16 * more), 0x55, dtype=torch.uint8, device="cuda"),
            torch.full((rows + 1, B.mv_f8_row_scales(n) + 4 * more), 0x55, dtype=torch.uint8, device="cuda"))


def check_codes(codes, scales, x, rows, n):
    want, want_scales = R.encode(x)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    blocks = R.blocks_of(n)
    assert np.array_equal(s[:rows, :blocks], want_scales)
    assert np.array_equal(c[:rows, : 128 * blocks], want), np.argwhere(c[:rows, : 128 * blocks] != want)[:4]
    assert (c[rows:] == 0x55).all() and (c[:, 128 * blocks:] == 0x55).all()
    assert (s[rows:] == 0x55).all() and (s[:, blocks:] == 0x55).all()
    return want, want_scales


def values(rng, rows, n):
    """Scales over decades, zeros, denormals, a row and a block of zeros."""
    x = rng.standard_normal((rows, n)) * np.exp(4.0 * rng.standard_normal((rows, n)))
    x *= 10.0 ** rng.integers(-20, 20, (rows, 1))
    x[rng.random((rows, n)) < 0.05] = 0.0
    x[rng.random((rows, n)) < 0.02] *= 1e-25
    if rows > 2:
        x[1] = 0.0
    x[0, :128] = -0.0
    return x.astype(np.float32)


SHAPES = [(1, 1), (1, 127), (3, 128), (5, 129), (2, 255), (33, 300), (16, 1000), (7, 2049), (1, 70_001), (300, 130)]


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_encode_decode(rows, n, src):
    rng = np.random.default_rng(rows * 100_003 + n)
    for lead, extra in ((0, 0), (1, 3)):
        x = place(values(rng, rows, n), TYPES[src], lead, extra)
        codes, scales = room(rows, n, more=extra)
        B.mv_f8_encode(x, codes[:rows], scales[:rows])
        want, want_scales = check_codes(codes, scales, x.float().cpu().numpy(), rows, n)
        held = R.values(want, want_scales, n)
        for dst in TYPES.values():
            out = torch.full((rows + 1, n + 3), 7.5, dtype=dst, device="cuda")
            B.mv_f8_decode(codes, scales, out[:rows, 1:n + 1])
            o = out.float().cpu().numpy()
            assert np.array_equal(o[:rows, 1:n + 1], torch.from_numpy(held.astype(np.float32)).to(dst).float().numpy())
            o[:rows, 1:n + 1] = 7.5
            assert (o == 7.5).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (7, 3), (31, 64), (127, 65), (128, 1), (129, 200), (300, 128), (513, 63), (1000, 77),
                                    (1, 500), (2049, 70)])
def test_columns(rows, n, src):
    rng = np.random.default_rng(rows * 1009 + n)
    for lead, extra in ((0, 0), (1, 3)):
        x = place(values(rng, rows, n), TYPES[src], lead, extra)
        codes, scales = room(n, rows, more=extra)
        B.mv_f8_encode_t(x, codes[:n], scales[:n])
        check_codes(codes, scales, np.ascontiguousarray(x.float().cpu().numpy().T), n, rows)


def whole_range():
    """Blocks whose largest value has each exponent of fp32, denormals among them, with a fraction on both sides of the next
    power; the others on the grid, at its middles and one unit beside them, over the whole grid."""
    grid = np.array([f * 2.0 ** -9 for f in range(8)] + [(8 + f) * 2.0 ** (e - 10) for e in range(1, 16) for f in range(8)][:-1])
    middles = (grid[1:] + grid[:-1]) / 2
    steps = np.concatenate([grid, middles]) / 448.0
    rows = []
    for e in range(-149, 128):
        for top in (1.0, 1.5, 1.75, 1.875):
            for shift in (-1, 0, 1):
                v = (2.0 ** e * top) * steps
                if shift and e > -100:
                    v = np.nextafter(v.astype(np.float32), np.float32(shift * 1e38)).astype(np.float64)
                v = np.concatenate([v, [2.0 ** e * top]])
                for at in range(0, len(v), 127):
                    row = np.resize(v[at:at + 127], 128)
                    row[127] = 2.0 ** e * top
                    rows.append(row * np.where(np.arange(128) % 2, -1, 1))
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[~np.isfinite(x)] = np.finfo(np.float32).max
    return x


@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_whole_range(src):
    x = whole_range()
    if src == "bf16":                                   # cut, so that nothing becomes infinite
        x = (x.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    d = place(x, TYPES[src], 0, 0)
    codes, scales = room(len(x), 128)
    B.mv_f8_encode(d, codes[:len(x)], scales[:len(x)])
    want, want_scales = check_codes(codes, scales, x, len(x), 128)
    out = torch.zeros((len(x), 128), device="cuda")
    B.mv_f8_decode(codes, scales, out)
    assert np.array_equal(out.cpu().numpy(), R.values(want, want_scales, 128).astype(np.float32))
    columns, column_scales = room(len(x), 128)
    B.mv_f8_encode_t(d.t().contiguous(), columns[:len(x)], column_scales[:len(x)])
    assert torch.equal(columns, codes) and torch.equal(column_scales[:, :1], scales[:, :1])


def test_every_code_and_scale_is_read():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    codes[127] = codes[255] = 0
    codes = codes.view(1, 256).expand(256, 256).contiguous()
    scales = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].expand(256, 4).contiguous()
    out = torch.zeros((256, 256), device="cuda")
    B.mv_f8_decode(codes, scales, out)
    with np.errstate(over="ignore"):
        want = R.values(codes.cpu().numpy(), scales.cpu().numpy()[:, :2], 256).astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)


def test_nan_and_infinity_take_their_block():
    x = np.ones((3, 400), np.float32)
    x[0, 140], x[1, 5], x[2, 399] = np.nan, np.inf, -np.inf
    for dtype in TYPES.values():
        d = place(x, dtype, 0, 0)
        codes, scales = room(3, 400)
        B.mv_f8_encode(d, codes[:3], scales[:3])
        check_codes(codes, scales, x, 3, 400)
        out = torch.zeros((3, 400), device="cuda")
        B.mv_f8_decode(codes, scales, out)
        lost = np.zeros((3, 400), bool)
        lost[0, 128:256] = lost[1, :128] = lost[2, 384:] = True
        assert np.array_equal(np.isnan(out.cpu().numpy()), lost) and (out.cpu().numpy()[~lost] == 1.0).all()
        codes_t, scales_t = room(400, 3)
        B.mv_f8_encode_t(d, codes_t[:400], scales_t[:400])
        check_codes(codes_t, scales_t, np.ascontiguousarray(x.T), 400, 3)


def test_long_rows_beyond_32_bits():
    """2^32 + 128 values in two rows: bytes and elements beyond 32 bits of offset."""
    n = (1 << 31) - 128
    x = torch.zeros((2, n), dtype=torch.bfloat16, device="cuda")
    x[1, n - 1], x[1, 7], x[0, n - 129] = 6.0, -3.0, 1.5
    codes = torch.zeros((2, B.mv_f8_row_bytes(n)), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((2, B.mv_f8_row_scales(n)), dtype=torch.uint8, device="cuda")
    B.mv_f8_encode(x, codes, scales)
    out = torch.full((2, n), 9.0, dtype=torch.bfloat16, device="cuda")
    B.mv_f8_decode(codes, scales, out)
    assert torch.equal(out, x)


def test_other_stream_and_graph():
    x = place(values(np.random.default_rng(4), 6, 5000), torch.float32, 0, 0)
    codes, scales = room(6, 5000)
    out, ref = torch.zeros((6, 5000), device="cuda"), torch.zeros((6, 5000), device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    B.mv_f8_encode(x, codes[:6], scales[:6], stream=s)
    B.mv_f8_decode(codes, scales, ref, stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.mv_f8_encode(x, codes[:6], scales[:6])
        B.mv_f8_decode(codes, scales, out)
    for _ in range(3):
        out.zero_()
        codes.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        x.neg_()
        B.mv_f8_encode(x, codes[:6], scales[:6])
        B.mv_f8_decode(codes, scales, ref)


def test_python_refusals():
    x = torch.zeros((4, 300), device="cuda")
    codes, scales = room(4, 300)
    for bad in (lambda: B.mv_f8_encode(x.half(), codes, scales), lambda: B.mv_f8_encode(x[:, ::2], codes, scales),
                lambda: B.mv_f8_encode(x, codes[:3], scales), lambda: B.mv_f8_encode(x, codes[:, :368], scales),
                lambda: B.mv_f8_encode(x, codes, scales[:, :3]), lambda: B.mv_f8_encode(x, codes.cpu(), scales),
                lambda: B.mv_f8_encode(x, codes.view(torch.int32), scales),
                lambda: B.mv_f8_encode_t(x, codes[:, :100], scales), lambda: B.mv_f8_decode(codes, scales, x.t())):
        with pytest.raises(ValueError):
            bad()
