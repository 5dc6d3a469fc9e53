"""Microscaled 4-bit tensors, norms and caches, restated plainly in numpy: float64 wherever a definition does not name a
narrower type.  Inputs are float64 arrays that hold float32, bfloat16 or float16 values exactly.

The element type is the (4, 1) type of Section 2.1 with its value taken in halves (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6),
pinned against oracle/dynfloat.py in tests/test_oracle_mx.py; conversion as there: nearest, ties to the even pattern, saturating,
NaN to code 0, never a negative zero.  One scale 2^(s - 127) per block of 32 values.
"""
import numpy as np

from oracle import dynfloat as df

BLOCK = 32
VALUES = np.array([float(df.decode_sign_magnitude(c, 4, 1)) / 2 for c in range(8)])


def _exponent(top, largest):
    """Smallest whole e with largest * 2^e >= top > 0, by trial."""
    e = int(np.floor(np.log2(top / largest))) - 1
    while np.ldexp(largest, e) < top:
        e += 1
    return e


def _top(x):
    a = np.abs(np.asarray(x, np.float64))
    a = a[np.isfinite(a)]
    return float(a.max()) if a.size else 0.0


def mx_exponent(block, rule):
    top = _top(block)
    if top == 0.0:
        return 0
    e = _exponent(top, 6.0) if rule == "cover" else int(np.frexp(top)[1]) - 1 - 2
    return max(e, -127)


def i8_exponent(group):
    top = _top(group)
    return 0 if top == 0.0 else max(_exponent(top, 127.0), -126)


def nearest_code(a):
    """Magnitudes (finite or inf) -> codes 0..7."""
    a = np.minimum(a, VALUES[-1])
    hi = np.clip(np.searchsorted(VALUES, a, side="left"), 1, 7)
    up, down = VALUES[hi] - a, a - VALUES[hi - 1]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)


def mx_quantize(x, rule="cover"):
    """[rows, K] -> codes [rows, blocks * 32] (one a byte), scale bytes [rows, blocks]."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    blocks = -(-K // BLOCK)
    codes, scales = np.zeros((rows, blocks * BLOCK), np.uint8), np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            v = x[r, b * BLOCK:(b + 1) * BLOCK]
            e = mx_exponent(v, rule)
            a = np.where(np.isnan(v), 0.0, np.abs(v)) * 2.0**-e
            c = nearest_code(a)
            codes[r, b * BLOCK:b * BLOCK + v.size] = np.where((v < 0) & (c > 0), c + 8, c)
            scales[r, b] = e + 127
    return codes, scales


def mx_values(codes, scales, K):
    sign = np.where(codes & 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (sign * VALUES[codes & 7] * np.repeat(power, BLOCK, axis=1))[:, :K]


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    out = np.empty((packed.shape[0], packed.shape[1] * 2), np.uint8)
    out[:, 0::2], out[:, 1::2] = packed & 15, packed >> 4
    return out


def to_tiles(scales):
    """Scale bytes [rows, blocks] -> tiles of 128 rows x 4 blocks, filled up with 127."""
    rows, blocks = scales.shape
    tr, tb = -(-rows // 128), -(-blocks // 4)
    out = np.full(tr * tb * 512, 127, np.uint8)
    for r in range(rows):
        for b in range(blocks):
            out[((r // 128) * tb + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4] = scales[r, b]
    return out


def i8_codes(y, e):
    """Values -> int8 at exponent e: nearest, ties to even, +-127, NaN to 0."""
    y = np.asarray(y, np.float64)
    return np.clip(np.rint(np.where(np.isnan(y), 0.0, y) * 2.0**-e), -127, 127).astype(np.int8)


def linear(x, w, bias=None, relu=False):
    y = x @ w.T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return np.maximum(y, 0.0) if relu else y


def rmsnorm(h, gain, eps):
    """h, gain float64 holding their type's values -> (y as defined: r and the two products rounded to float32; y in
    float64 throughout)."""
    with np.errstate(all="ignore"):
        m = (h * h).sum(-1, keepdims=True) / h.shape[1] + eps
        r = 1.0 / np.sqrt(m)
        y32 = (h.astype(np.float32) * r.astype(np.float32)) * gain.astype(np.float32)
        return y32.astype(np.float64), h * r * gain
