"""Microscaled 4-bit values in numpy, from the definition in include/mv.h, in 64 bits."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDDLES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def blocks_of(n):
    return (n + 31) // 32


def encode(x):
    """(places with the sign as bit 3: rows x 32 blocks, scale bytes: rows x blocks) of float32 rows."""
    rows, n = x.shape
    v = np.zeros((rows, 32 * blocks_of(n)))
    with np.errstate(invalid="ignore"):
        v[:, :n] = x.astype(np.float64)
    v = v.reshape(rows, -1, 32)
    bad = ~np.isfinite(v).all(2)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(2))
    s = np.maximum(np.frexp(top)[1] - 1 - 2, -127)
    s = np.where(top == 0.0, -127, s)
    v = np.where(bad[:, :, None], 0.0, v)
    a = np.abs(v) / np.exp2(s.astype(np.float64))[:, :, None]
    place = np.zeros(v.shape, np.int64)
    for i, mid in enumerate(MIDDLES):
        place += (a > mid) if i % 2 == 0 else (a >= mid)
    codes = place | (np.signbit(v).astype(np.int64) << 3)
    scales = np.where(bad, 255, s + 127).astype(np.uint8)
    return codes.reshape(rows, -1), scales


def pack(codes):
    """32-bit words of codes."""
    c = codes.reshape(codes.shape[0], -1, 8).astype(np.uint64)
    return (c << (4 * np.arange(8, dtype=np.uint64))).sum(2).astype(np.uint32)


def unpack(words):
    return ((words[:, :, None] >> (4 * np.arange(8, dtype=np.uint32))) & 15).reshape(words.shape[0], -1).astype(np.int64)


def values(codes, scales, n):
    """What codes and scales stand for, in 64 bits."""
    s = scales.astype(np.int64)[:, : blocks_of(n)] - 127
    p = np.where(s == 128, np.nan, np.exp2(s.astype(np.float64)))
    q = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    q = q.reshape(codes.shape[0], -1, 32) * p[:, :, None]
    return q.reshape(codes.shape[0], -1)[:, :n]


def held(x):
    codes, scales = encode(x)
    return values(codes, scales, x.shape[1])
