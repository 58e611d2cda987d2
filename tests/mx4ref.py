"""The microscaled 4-bit format in numpy, in 64 bits, from its definition; and exact products."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(k):
    return -(-k // 128) * 128


def quantize(x):
    """[rows, K] floats -> codes [rows, Kp / 2], scales [rows, Kp / 32] (uint8)."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    b = np.zeros((rows, padded(k)))
    b[:, :k] = x
    b = b.reshape(rows, -1, 32)
    top = np.abs(b).max(2)
    bad = ~np.isfinite(b).all(2)
    _, e = np.frexp(np.where(bad | (top == 0), 1.0, top))          # top = m 2^e, m in [0.5, 1)
    e = np.maximum(np.where(top == 0, -127, e - 3), -127)
    a = np.where(bad[:, :, None], 0.0, np.abs(b)) / np.exp2(e.astype(np.float64))[:, :, None]
    d = np.abs(a[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    tie = d == near
    # of two equally near codes the even one
    code = np.where(tie.sum(-1) > 1, (tie * np.arange(8) * (np.arange(8) % 2 == 0)).max(-1), d.argmin(-1))
    code = np.where(bad[:, :, None], 0, code + 8 * np.signbit(np.where(bad[:, :, None], 0.0, b)))
    code = code.reshape(rows, -1).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales


def values(codes, scales, k=None):
    """float64 [rows, K]"""
    c = np.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = (v.reshape(len(codes), -1, 32) * s[:, :, None]).reshape(len(codes), -1)
    return v if k is None else v[:, :k]


def held(rng, rows, k, lo=126, hi=128):
    """Random held rows, zero codes and scales behind K.  With scales in 126..128 a product of two values is a whole
    multiple of 2^-4 and at most 144: sums of 7000 of them are exact in float32 in any order."""
    kp = padded(k)
    code = rng.integers(0, 16, (rows, kp)).astype(np.uint8)
    code[:, k:] = 0
    scales = rng.integers(lo, hi + 1, (rows, kp // 32)).astype(np.uint8)
    scales[:, -(-k // 32):] = 0
    return code[:, 0::2] | (code[:, 1::2] << 4), scales


def ternary(rng, n, k, keep=0.6):
    return ((rng.random((n, k)) < keep) * rng.choice(np.array([-1, 1]), (n, k))).astype(np.int8)
