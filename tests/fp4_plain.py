"""Plain 64-bit forms of the operators over 4-bit rows, the rotation and the norms, for the tests: numpy, written from the
definitions, sharing nothing with the library."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LARGEST = {0: 140, 1: 252}  # scale bytes of blocks of fp16 / bf16 numbers
HALF_STEP = {0: 2.0 ** -11, 1: 2.0 ** -8, 2: 2.0 ** -24}  # of S3_F16, S3_BF16, S3_F32, relative


def row_bytes(heads, d):
    return -(-(heads * (d // 2 + d // 32)) // 16) * 16


def to_rows(x, act):
    """float64 [n][heads][d] -> stored rows uint8 [n][row_bytes]."""
    n, heads, d = x.shape
    b = x.reshape(n, heads, d // 32, 32)
    ok = np.isfinite(b).all(-1)
    most = np.where(ok, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1), 1.0)
    byte = np.full(most.shape, 1)
    for k in range(2, LARGEST[act] + 1):  # the least power of two under which the largest is below 7
        byte[most >= 7.0 * 2.0 ** (k - 1 - 127)] = k
    y = np.where(ok[..., None], b, 0.0) / 2.0 ** (byte[..., None] - 127.0)
    off = np.abs(np.abs(y)[..., None] - VALUES)
    code = np.argmin(off, -1)
    tie = np.isclose(np.take_along_axis(off, np.minimum(code + 1, 7)[..., None], -1)[..., 0], off.min(-1), rtol=0, atol=0)
    code = np.where(tie & (code % 2 == 1) & (code < 7), code + 1, code)  # a tie goes to the even code
    code = np.where(np.signbit(y) & ok[..., None], code + 8, code).astype(np.uint8).reshape(n, heads, d)
    out = np.zeros((n, row_bytes(heads, d)), np.uint8)
    packed = code[..., 0::2] | code[..., 1::2] << 4
    out[:, :heads * d // 2] = packed.reshape(n, heads * d // 2)
    out[:, heads * d // 2:heads * (d // 2 + d // 32)] = np.where(ok, byte, 255).astype(np.uint8).reshape(n, heads * d // 32)
    return out


def from_rows(rows, heads, d):
    """Stored rows -> float64 [n][heads][d]."""
    n = rows.shape[0]
    codes = rows[:, :heads * d // 2]
    scales = rows[:, heads * d // 2:heads * (d // 2 + d // 32)].reshape(n, heads, d // 32).astype(np.float64)
    c = np.stack((codes & 15, codes >> 4), -1).reshape(n, heads, d // 32, 32)
    x = np.where(c >= 8, -VALUES[c % 8], VALUES[c % 8])
    return (x * np.where(scales == 255, np.nan, 2.0 ** (scales - 127))[..., None]).reshape(n, heads, d)


def attention(q, k, v, scale=None):
    """q [Hq][d], k, v [L][Hkv][d] float64 -> (out, bound of a 32-bit computation's error) [Hq][d].
    The bound, element by element: a score is a sum of d products in fp32, off by at most (d + 4) * 2^-24 of the sum of their
    magnitudes (times the scale; scale, log2(e) and the subtraction of the reference add roundings of the score itself); a weight
    is off by that and 2^-22 (exp2), as are both sums, whose additions are off by L * 2^-24 at most."""
    hq, d = q.shape
    L, hkv, _ = k.shape
    if L == 0:
        return np.zeros((hq, d)), np.zeros((hq, d))
    scale = d ** -0.5 if scale is None else scale
    out, bound = np.empty((hq, d)), np.empty((hq, d))
    for h in range(hq):
        kk, vv = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        s = kk @ q[h] * scale
        most = (np.abs(kk) @ np.abs(q[h])).max() * abs(scale)
        w = np.exp(s - s.max())
        w /= w.sum()
        out[h] = w @ vv
        err = 2 * ((d + 4) * 2.0 ** -24 * most + 4 * 2.0 ** -24 * (np.abs(s).max() + 8) + 2.0 ** -22 + (L + 64) * 2.0 ** -24)
        bound[h] = err * (w @ np.abs(vv))
    return out, bound


def allowed(out, bound, magnitude_parts, out_dtype):
    """Bound of an output in out_dtype; magnitude_parts: |out| and sum of w |v| come from the same weights, whose two-part form (16-bit
    outputs) is off by 2^-16 of a weight (2^-17, and the sum's own)."""
    more = 0.0 if out_dtype == 2 else 2.0 ** -16
    return bound + more * magnitude_parts + HALF_STEP[out_dtype] * (np.abs(out) + bound) + 1e-30 + (2.0 ** -25 if out_dtype == 0 else 0.0)


def rotate(x, weight, rotary, interleaved, angle, eps):
    """x [n][heads][d] float64, angle [n][rotary/2] -> (y, magnitudes that an error is relative to)."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    y, mag = x.copy(), np.abs(x)
    half = rotary // 2
    i = np.arange(half) * (2 if interleaved else 1)
    j = i + (1 if interleaved else half)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    mag[..., i] = mag[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return y, mag
