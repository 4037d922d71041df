"""Plain restatement of the 4-bit formats with numpy, value by value from the definitions in include/signsgd.h."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"mx": 32, "nv": 16}


def e4m3_values():
    v = np.empty(127)
    for b in range(127):
        e, f = b >> 3, b & 7
        v[b] = f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
    return v


E4M3 = e4m3_values()


def nearest_even(values, y):
    """Index of the entry of `values` nearest to y, a tie to the even index, beyond the last to the last."""
    hi = np.clip(np.searchsorted(values, y), 1, len(values) - 1)
    lo = hi - 1
    dl, dh = y - values[lo], values[hi] - y
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(up, hi, lo)


def tensor_scale(amax):
    if not np.isfinite(amax) or amax <= 0:
        return 1.0
    t = int(np.floor(np.log2(amax / 2688.0))) - 1
    while 2688.0 * 2.0 ** t < amax:
        t += 1
    return 2.0 ** min(120, max(-100, t))


def quantise(x, fmt, amax=None):
    """codes [rows][cols] (0..15), scale bytes [rows][blocks], tensor scale of a float32 array that holds x exactly."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    b = BLOCK[fmt]
    nb = -(-cols // b)
    p = np.zeros((rows, nb * b), dtype=np.float32)
    p[:, :cols] = x
    p = p.reshape(rows, nb, b)
    top = np.abs(p).max(axis=2).astype(np.float64)
    bad = ~np.isfinite(top)
    safe = np.where(bad, 1.0, top)
    if fmt == "mx":
        ts = 1.0
        _, e = np.frexp(safe)
        e = np.where(safe > 0, np.maximum(e - 3, -127), -127)
        S = 2.0 ** e.astype(np.float64)
        byte = np.where(bad, 255, e + 127)
    else:
        all_top = np.abs(x).max() if amax is None else amax
        ts = tensor_scale(float(all_top)) if x.size else 1.0
        third = (np.minimum(safe / ts, 3e38).astype(np.float32) / np.float32(6.0)).astype(np.float64)
        byte = np.maximum(nearest_even(E4M3, np.minimum(third, 448.0)), 1)
        S = E4M3[byte] * ts
        byte = np.where(bad, 0x7F, byte)
    with np.errstate(all="ignore"):
        q = (p.astype(np.float64) / S[:, :, None]).astype(np.float32).astype(np.float64)   # the fp32 quotient
        mag = nearest_even(LEVELS, np.minimum(np.abs(np.where(np.isfinite(q), q, 0.0)), 100.0))
        mag = np.where(np.isinf(q), 7, mag)
    code = mag + 8 * np.signbit(p)
    code = np.where(bad[:, :, None], 0, code)
    return code.reshape(rows, nb * b)[:, :cols].astype(np.uint8), byte.astype(np.uint8), ts


def values(code, byte, ts, fmt):
    """float64 values of codes and scale bytes."""
    v = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    if fmt == "mx":
        s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    else:
        s = np.where(byte == 0x7F, np.nan, E4M3[np.minimum(byte, 126)]) * ts
    return v * np.repeat(s, BLOCK[fmt], axis=1)[:, :code.shape[1]]


def pack_codes(code):
    rows, cols = code.shape
    p = np.zeros((rows, -(-cols // 32) * 32), dtype=np.uint8)
    p[:, :cols] = code
    return (p[:, 0::2] | (p[:, 1::2] << 4)).astype(np.uint8)


def pack_scales(byte):
    rows, nb = byte.shape
    tk = -(-nb // 4)
    out = np.zeros(-(-rows // 128) * tk * 512, dtype=np.uint8)
    r, k = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[((r // 128) * tk + k // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + k % 4] = byte
    return out
