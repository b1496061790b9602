"""8-bit values by blocks of 128 in numpy, from the definition in include/mv.h, in 64 bits."""
import numpy as np


def blocks_of(n):
    return (n + 127) // 128


def encode(x):
    """(codes: rows x 128 blocks uint8, scale bytes: rows x blocks) of float32 rows."""
    rows, n = x.shape
    v = np.zeros((rows, 128 * blocks_of(n)))
    with np.errstate(invalid="ignore"):
        v[:, :n] = x.astype(np.float64)
    v = v.reshape(rows, -1, 128)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[:, :, None], 0.0, v)
    top = np.abs(v).max(2)
    s = np.full(top.shape, -127)
    for e in range(-126, 121):                          # the smallest s with top <= 448 * 2^s
        s = np.where(top > 448.0 * 2.0 ** (e - 1), e, s)
    a = np.abs(v) / np.exp2(s.astype(np.float64))[:, :, None]
    e = np.maximum(np.frexp(a)[1] - 1, -6)
    f = np.rint(a / np.exp2(e - 3.0)).astype(np.int64)  # in eighths of 2^e: 8 .. 16, or below 8 where e is -6; ties to even
    e, f = np.where(f == 16, e + 1, e), np.where(f == 16, 8, f)
    codes = np.where(f >= 8, (e + 7) * 8 + f - 8, f) | (np.signbit(v).astype(np.int64) << 7)
    return codes.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, s + 127).astype(np.uint8)


def values(codes, scales, n):
    """What codes and scales stand for, in 64 bits."""
    c = codes.astype(np.int64)
    e, f = c >> 3 & 15, c & 7
    q = np.where(e == 0, f * 2.0 ** -9, (8 + f) * np.exp2(e - 10.0)) * np.where(c & 128, -1.0, 1.0)
    s = scales.astype(np.int64)[:, : codes.shape[1] // 128] - 127
    p = np.where(s == 128, np.nan, np.exp2(s.astype(np.float64)))
    return (q.reshape(codes.shape[0], -1, 128) * p[:, :, None]).reshape(codes.shape[0], -1)[:, :n]


def held(x):
    return values(*encode(x), x.shape[1])
