"""CPU oracle of the 8-bit layer: e4m3 by its table of values, the block quantizer, the product in fp64; test infrastructure only."""
import numpy as np


def _values():
    """The 127 non-negative e4m3 values by code: 4 exponent bits (bias 7), 3 mantissa bits, no infinity, 0x7f is NaN."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


VALUES = _values()


def decode(codes):
    codes = np.asarray(codes, np.uint8)
    mag = codes & 0x7f
    v = np.where(mag == 0x7f, np.nan, VALUES[np.minimum(mag, 126)])
    return np.where(codes & 0x80, -v, v)


def encode(v):
    """Nearest value, ties to the even code; |v| <= 448 or not finite (NaN)."""
    v = np.asarray(v, np.float64)
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    assert (a <= 448).all()
    hi = np.searchsorted(VALUES, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - VALUES[lo], VALUES[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isfinite(v), code, 0x7f)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def block_scale(block):
    a = np.abs(np.asarray(block, np.float64))
    top = a[np.isfinite(a)].max(initial=0.0)
    if top == 0:
        return 1.0
    e = -126
    while 448 * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def quantize(W, rows=128):
    """Blocks of `rows` x 128 (the last ones ragged): codes [N][K], scales [ceil(N/rows)][ceil(K/128)]."""
    W = np.asarray(W, np.float64)
    N, K = W.shape
    codes, scales = np.zeros((N, K), np.uint8), np.zeros((-(-N // rows), -(-K // 128)))
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            b = W[rows * i:rows * (i + 1), 128 * j:128 * (j + 1)]
            scales[i, j] = block_scale(b)
            codes[rows * i:rows * (i + 1), 128 * j:128 * (j + 1)] = encode(b / scales[i, j])
    return codes, scales


def _spread(scales, N, K):
    return np.repeat(np.repeat(np.asarray(scales, np.float64), 128, 0)[:N], 128, 1)[:, :K]


def linear(x, codes, scales):
    """y [M][N] in fp64, and the sum of the magnitudes of its terms (what rounding errors of a sum are relative to)."""
    x = np.asarray(x, np.float64)
    N, K = codes.shape
    xc, xs = quantize(x, rows=1)
    xq = decode(xc) * np.repeat(xs, 128, 1)[:, :K]
    w = decode(codes) * _spread(scales, N, K)
    return xq @ w.T, np.abs(xq) @ np.abs(w).T
