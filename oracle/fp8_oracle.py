"""fp64 CPU oracle for rows held in 8 bits and the projections of them.

TEST INFRASTRUCTURE ONLY.  Nothing on the product path may import this file; it shares no code with the
GPU library and imports nothing from the package.

The format (include/aeris_fp8.h states it): e4m3 values, and one power-of-two scale for each block of 128
columns of a row (a shorter one at its end).  e4m3 is enumerated here from its definition (sign, four exponent
bits of bias 7, three mantissa bits, subnormal steps of 2^-9, the codes 0x7f and 0xff not a number) and a value
is rounded by looking its two neighbours up, ties to the code with an even last bit.

Parity pins: tests/test_fp8_host.py.
"""
import numpy as np

BLOCK = 128
LEAST_EXPONENT = -126


def _table():
    codes = np.arange(127)                                # non-negative numbers
    exponent, mantissa = codes >> 3, codes & 7
    return np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent - 10.0))


TABLE = _table()


def encode(v):
    """Nearest e4m3 code of |v| <= 448, ties to the even code; 0x7f (with the sign bit free) where not finite."""
    v = np.asarray(v, dtype=np.float64)
    size = np.abs(np.where(np.isfinite(v), v, 0.0))
    assert size.max(initial=0.0) <= 448.0
    hi = np.searchsorted(TABLE, size)                     # TABLE[hi - 1] < size <= TABLE[hi]
    lo = np.maximum(hi - 1, 0)
    below, above = size - TABLE[lo], TABLE[hi] - size
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isfinite(v), code | (np.signbit(v) << 7), 0x7f)
    return code.astype(np.uint8)


def decode(code):
    code = np.asarray(code)
    size = np.where((code & 127) == 127, np.nan, TABLE[np.minimum(code & 127, 126)])
    return np.where(code & 128, -size, size)


def scale_pitch(cols):
    return -(-(-(-cols // BLOCK)) // 4) * 4


def quantize(x):
    """x [n, c] -> (codes uint8 [n, c], scale bytes uint8 [n, scale_pitch(c)])."""
    x = np.asarray(x, dtype=np.float64)
    n, c = x.shape
    codes = np.empty((n, c), dtype=np.uint8)
    scales = np.full((n, scale_pitch(c)), 127, dtype=np.uint8)
    for b in range(-(-c // BLOCK)):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        most = np.abs(np.where(np.isfinite(part), part, 0.0)).max(axis=1)
        e = np.full(n, LEAST_EXPONENT)
        while True:                                       # upwards from the smallest
            over = most > 448.0 * 2.0 ** e.astype(np.float64)
            if not over.any():
                break
            e[over] += 1
        scales[:, b] = e + 127
        codes[:, b * BLOCK:(b + 1) * BLOCK] = encode(part / 2.0 ** e.astype(np.float64)[:, None])
    return codes, scales


def per_column(scales, cols):
    """2^e for every column."""
    return np.repeat(2.0 ** (np.asarray(scales, dtype=np.float64) - 127.0), BLOCK, axis=1)[:, :cols]


def dequantize(codes, scales):
    return decode(codes) * per_column(scales, codes.shape[1])


def round_trip(x):
    return dequantize(*quantize(x))


def linear_fwd(x, w):
    """x [n, c], w [f, c] -> x w^T."""
    return np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T


def linear_bwd(x, w_transposed, dy):
    """(dx, dw) of y = x w^T, with dy quantised by rows for dx alone; w_transposed [c, f]."""
    dy = np.asarray(dy, dtype=np.float64)
    return round_trip(dy) @ np.asarray(w_transposed, dtype=np.float64).T, dy.T @ np.asarray(x, dtype=np.float64)
