"""Microscaled 4-bit values against their definition in numpy (tests/mx_reference.py): codes, scales, residuals and what is
read back are exact."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2011_06495_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FILL = 0x5A


@pytest.fixture(autouse=True)
def say(request):
    print("[case] " + request.node.name, flush=True)


def place(x, dtype, lead, extra):
    """x on the device with `extra` more elements in a row, beginning `lead` elements behind an aligned address."""
    rows, n = x.shape
    buf = torch.zeros(rows * (n + extra) + lead, dtype=dtype, device="cuda")
    t = buf[lead:].view(rows, n + extra)[:, :n]
    t.copy_(torch.from_numpy(x))
    return t


def room(rows, n, more=0):
    """Codes and scales, filled, with `more` groups of four words and scales than a row needs."""
    codes = torch.full((rows + 1, B.mv_mx_row_words(n) + 4 * more), FILL, dtype=torch.int32, device="cuda")
    scales = torch.full((rows + 1, B.mv_mx_row_scales(n) + 4 * more), FILL, dtype=torch.uint8, device="cuda")
    return codes, scales


def check_codes(codes, scales, x, rows, n):
    want, want_scales = R.encode(x)
    c, s = codes.cpu().numpy().view(np.uint32), scales.cpu().numpy()
    words, blocks = B.mv_mx_row_words(n), R.blocks_of(n)
    assert np.array_equal(s[:rows, :blocks], want_scales)
    assert np.array_equal(c[:rows, :words], R.pack(want))
    assert (c[rows:] == FILL).all() and (c[:, words:] == FILL).all()
    assert (s[rows:] == FILL).all() and (s[:, blocks:] == FILL).all()
    return want, want_scales


def values(rng, rows, n):
    """Normal values over decades, with zeros, whole blocks of them, and ties of every kind."""
    x = rng.standard_normal((rows, n)) * np.exp(2.0 * rng.standard_normal((rows, n)))
    ties = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0], size=(rows, n))
    x = np.where(rng.random((rows, n)) < 0.3, ties * rng.choice([-1.0, 1.0], size=(rows, n)), x)
    for r in range(0, rows, 3):
        x[r, 32:64] = 0.0
    return x.astype(np.float32)


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (2, 8), (5, 31), (1, 32), (70, 33), (3, 64), (4, 65), (200, 100), (3, 1000),
                                    (2, 2049), (7, 2048), (1, 70_001)])
def test_encode_decode(rows, n, src):
    rng = np.random.default_rng(rows * 100_003 + n)
    for lead, extra in ((0, 0), (1, 3)):
        x = place(values(rng, rows, n), TYPES[src], lead, extra)
        x32 = x.float().cpu().numpy()
        codes, scales = room(rows, n, more=extra)
        resid = torch.full((rows + 1, n + 2), 7.5, device="cuda")
        B.mv_mx_encode(x, codes[:rows], scales[:rows], resid=resid[:rows, :n])
        want, want_scales = check_codes(codes, scales, x32, rows, n)
        held = R.values(want, want_scales, n)
        r = resid.cpu().numpy()
        assert np.array_equal(r[:rows, :n], (x32.astype(np.float64) - held).astype(np.float32))
        assert np.array_equal(r[:rows, :n].astype(np.float64), x32.astype(np.float64) - held)     # no rounding in it
        assert (r[rows:] == 7.5).all() and (r[:, n:] == 7.5).all()
        again, more = room(rows, n)
        B.mv_mx_encode(x, again[:rows], more[:rows])
        check_codes(again, more, x32, rows, n)
        for dst in TYPES.values():
            out = torch.full((rows + 1, n + 3), 7.5, dtype=dst, device="cuda")
            B.mv_mx_decode(codes, scales, out[:rows, 1:n + 1])
            o = out.float().cpu().numpy()
            assert np.array_equal(o[:rows, 1:n + 1], torch.from_numpy(held.astype(np.float32)).to(dst).float().numpy())
            o[:rows, 1:n + 1] = 7.5
            assert (o == 7.5).all()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (7, 3), (31, 64), (32, 65), (33, 1), (100, 200), (128, 128), (129, 63), (1000, 77),
                                    (1, 500), (2049, 70)])
def test_columns(rows, n, src):
    rng = np.random.default_rng(rows * 1009 + n)
    for lead, extra in ((0, 0), (1, 3)):
        x = place(values(rng, rows, n), TYPES[src], lead, extra)
        codes, scales = room(n, rows, more=extra)
        B.mv_mx_encode_t(x, codes[:n], scales[:n])
        check_codes(codes, scales, np.ascontiguousarray(x.float().cpu().numpy().T), n, rows)


def test_every_exponent_and_every_sixteenth():
    """Blocks whose largest value has each exponent of fp32, denormals among them, the others at the grid's middles, one unit
    beside them, and spread over [0, 8)."""
    rows = []
    for e in range(-149, 128):
        top = np.ldexp(1.0, e)
        step = np.concatenate([np.arange(16) / 16.0 + 0.0, [0.0625, 0.1875, 0.3125, 0.4375, 0.625, 0.875, 1.25]])
        v = top * step
        v = np.concatenate([v, np.nextafter(v[16:].astype(np.float32), np.float32(0)), [top]])
        rows.append(np.resize(v, 32) * np.where(np.arange(32) % 2, -1, 1))
        more = top * (1.0 + np.arange(32) / 32.0)                    # the largest, up to twice: cut at 6
        rows.append(more)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[~np.isfinite(x)] = np.finfo(np.float32).max
    d = place(x, torch.float32, 0, 0)
    codes, scales = room(len(x), 32)
    resid = torch.zeros((len(x), 32), device="cuda")
    B.mv_mx_encode(d, codes[:len(x)], scales[:len(x)], resid=resid)
    want, want_scales = check_codes(codes, scales, x, len(x), 32)
    held = R.values(want, want_scales, 32)
    assert np.array_equal(resid.cpu().numpy().astype(np.float64), x.astype(np.float64) - held)
    out = torch.zeros((len(x), 32), device="cuda")
    B.mv_mx_decode(codes, scales, out)
    assert np.array_equal(out.cpu().numpy().astype(np.float64), held)


def test_nan_and_infinity_take_their_block():
    x = np.ones((3, 100), np.float32)
    x[0, 40], x[1, 5], x[2, 99] = np.nan, np.inf, -np.inf
    d = place(x, torch.float32, 0, 0)
    codes, scales = room(3, 100)
    resid, out, mean = torch.zeros((3, 100), device="cuda"), torch.zeros((3, 100), device="cuda"), torch.zeros(100, device="cuda")
    B.mv_mx_encode(d, codes[:3], scales[:3], resid=resid)
    check_codes(codes, scales, x, 3, 100)
    B.mv_mx_decode(codes, scales, out)
    B.mv_mx_aggregate(codes[:3], scales[:3], None, mean)
    lost = np.zeros((3, 100), bool)
    lost[0, 32:64] = lost[1, :32] = lost[2, 96:] = True
    assert np.array_equal(np.isnan(out.cpu().numpy()), lost) and np.array_equal(np.isnan(resid.cpu().numpy()), lost)
    assert (out.cpu().numpy()[~lost] == 1.0).all()
    assert np.array_equal(np.isnan(mean.cpu().numpy()), lost.any(0))
    codes_t, scales_t = room(100, 3)
    B.mv_mx_encode_t(d, codes_t[:100], scales_t[:100])
    check_codes(codes_t, scales_t, np.ascontiguousarray(x.T), 100, 3)


def test_residual_in_place():
    x = values(np.random.default_rng(2), 5, 333)
    d = place(x, torch.float32, 1, 2)
    codes, scales = room(5, 333)
    B.mv_mx_encode(d, codes[:5], scales[:5], resid=d)
    want, want_scales = check_codes(codes, scales, x, 5, 333)
    assert np.array_equal(d.cpu().numpy().astype(np.float64), x.astype(np.float64) - R.values(want, want_scales, 333))


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rows,n", [(1, 1), (2, 7), (7, 8), (8, 33), (9, 1000), (33, 4097), (300, 65)])
def test_aggregate(rows, n, weighted):
    """The sum is formed in fp32 in the rows' order, each product rounded: numpy does the same."""
    rng = np.random.default_rng(rows + n)
    x = values(rng, rows, n)
    codes, scales = room(rows, n)
    B.mv_mx_encode(place(x, torch.float32, 0, 0), codes[:rows], scales[:rows])
    held = R.held(x).astype(np.float32)
    w = rng.random(rows).astype(np.float32) if weighted else None
    agg = torch.full((n + 1,), 7.5, device="cuda")
    B.mv_mx_aggregate(codes[:rows], scales[:rows], torch.from_numpy(w).cuda() if weighted else None, agg[:n])
    want = np.zeros(n, np.float32)
    for r in range(rows):
        want += held[r] * w[r] if weighted else held[r]
    if not weighted:
        want *= np.float32(1.0) / np.float32(rows)
    got = agg.cpu().numpy()
    assert np.array_equal(got[:n], want) and got[n] == 7.5


def test_error_feedback_loses_nothing_over_steps():
    """Sending x + buffer each step and keeping the residual: what was sent adds up to what came in, less the buffer."""
    rng = np.random.default_rng(8)
    rows, n = 4, 500
    buf = torch.zeros((rows, n), device="cuda")
    sent, came = np.zeros((rows, n)), np.zeros((rows, n))
    codes, scales = room(rows, n)
    out = torch.zeros((rows, n), device="cuda")
    for _ in range(20):
        x = (rng.integers(-255, 256, (rows, n)) / 512.0).astype(np.float32)      # sums stay exact in fp32
        buf += torch.from_numpy(x).cuda()
        B.mv_mx_encode(buf, codes[:rows], scales[:rows], resid=buf)
        B.mv_mx_decode(codes, scales, out)
        sent += out.cpu().numpy()
        came += x
    assert np.array_equal(sent + buf.cpu().numpy(), came)


def test_long_rows_beyond_32_bits():
    """2^31 + 64 values in two rows: words and bytes beyond 32 bits of offset."""
    n = (1 << 30) + 32
    x = torch.zeros((2, n), dtype=torch.bfloat16, device="cuda")
    x[1, n - 1], x[1, 7], x[0, n - 33] = 6.0, -3.0, 1.5
    codes = torch.zeros((2, B.mv_mx_row_words(n)), dtype=torch.int32, device="cuda")
    scales = torch.zeros((2, B.mv_mx_row_scales(n)), dtype=torch.uint8, device="cuda")
    B.mv_mx_encode(x, codes, scales)
    out = torch.full((2, n), 9.0, dtype=torch.bfloat16, device="cuda")
    B.mv_mx_decode(codes, scales, out)
    assert torch.equal(out, x)


def test_other_stream_and_graph():
    x = place(values(np.random.default_rng(4), 6, 5000), torch.float32, 0, 0)
    codes, scales = room(6, 5000)
    agg = torch.zeros(5000, device="cuda")
    ref = torch.zeros(5000, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    B.mv_mx_encode(x, codes[:6], scales[:6], stream=s)
    B.mv_mx_aggregate(codes[:6], scales[:6], None, ref, stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.mv_mx_encode(x, codes[:6], scales[:6])
        B.mv_mx_aggregate(codes[:6], scales[:6], None, agg)
    for i in range(3):
        agg.zero_()
        codes.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(agg, ref)
        x.mul_(2.0)
        ref.mul_(2.0)


def test_python_refusals():
    x = torch.zeros((4, 100), device="cuda")
    codes, scales = room(4, 100)
    for bad in (lambda: B.mv_mx_encode(x.half(), codes, scales), lambda: B.mv_mx_encode(x[:, ::2], codes, scales),
                lambda: B.mv_mx_encode(x, codes[:3], scales), lambda: B.mv_mx_encode(x, codes[:, :12], scales),
                lambda: B.mv_mx_encode(x, codes, scales[:, :2]), lambda: B.mv_mx_encode(x, codes, scales, resid=x[:, :99]),
                lambda: B.mv_mx_encode(x, codes, scales, resid=x.bfloat16()), lambda: B.mv_mx_encode(x, codes.cpu(), scales),
                lambda: B.mv_mx_encode_t(x, codes[:, :4], scales), lambda: B.mv_mx_decode(codes, scales, x.t()),
                lambda: B.mv_mx_aggregate(codes, scales, x[0, :4].double(), x[0]),
                lambda: B.mv_mx_aggregate(codes, scales, x[0, :3], x[0]),
                lambda: B.mv_mx_aggregate(codes, scales, None, x[:, 0])):
        with pytest.raises(ValueError):
            bad()
