"""The 4-bit formats restated in numpy: codes are decided in float32 with IEEE division, as the definition says; values are float64."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NV, MX = 0, 1


def group(fmt):
    return 16 if fmt == NV else 32


def _e4m3_table():
    return np.array([(b & 7) * 2.0 ** -9 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) for b in range(127)])


E4M3 = _e4m3_table()


def e4m3_byte(x):
    """Nearest E4M3 value of x >= 0 (float32), ties to the even byte, saturating."""
    x = np.minimum(x.astype(np.float64), 448.0)
    hi = np.clip(np.searchsorted(E4M3, x), 1, 126)
    lo = hi - 1
    dl, dh = x - E4M3[lo], E4M3[hi] - x
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)


def scale_value(b, fmt):
    if fmt == NV:
        return np.where(b == 127, np.nan, E4M3[np.minimum(b, 126)])
    return np.where(b == 255, np.nan, 2.0 ** (b.astype(np.float64) - 127))


def quantize(x, fmt, t=1.0):
    """x float32 [..., d] -> codes uint8 [..., d] (four bits each), scale bytes [..., d / group], values float64 [..., d]."""
    t = np.float32(t)
    g = x.astype(np.float32).reshape(*x.shape[:-1], -1, group(fmt))
    with np.errstate(all="ignore"):
        a = np.abs(g).max(-1)
        bad = ~np.isfinite(g).all(-1)
        if fmt == NV:
            b = e4m3_byte(np.where(bad, 0, a / np.float32(t * np.float32(6))))
            b = np.where(bad, 127, b).astype(np.uint8)
        else:
            q = np.where(bad, 1, a / t).astype(np.float32)
            e = np.where(q > 0, np.frexp(np.where((q > 0) & np.isfinite(q), q, 1))[1] - 1, -127) - 2
            e = np.where(np.isinf(q), 127, e)
            b = np.where(bad, 255, np.clip(e, -127, 127) + 127).astype(np.uint8)
        s = scale_value(b, fmt).astype(np.float32)
        u = (s * t).astype(np.float32)
        y = (np.abs(g) / u[..., None]).astype(np.float32)
        c = (y > 0.25) + (y >= 0.75).astype(int) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
        c = np.where((s > 0)[..., None], c + 8 * (g < 0), 0).astype(np.uint8)
    c = c.reshape(x.shape)
    return c, b, values(c, b, fmt, t)


def values(codes, scale_bytes, fmt, t=1.0):
    """What codes stand for, in 64 bits."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    v = v.reshape(*codes.shape[:-1], -1, group(fmt)) * scale_value(scale_bytes, fmt)[..., None]
    return v.reshape(codes.shape) * float(np.float32(t))


def unpack(b):
    return np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], -1)


def pack(c):
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def tile_scales(b):
    """Row-major scale bytes [rows, groups] in the product's layout, byte by byte from its formula."""
    rows, groups = b.shape
    g4 = -(-groups // 4)
    out = np.zeros(-(-rows // 128) * g4 * 512, np.uint8)
    r, g = np.meshgrid(np.arange(rows), np.arange(groups), indexing="ij")
    out[((r // 128) * g4 + g // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + g % 4] = b
    return out
