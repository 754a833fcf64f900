"""Microscaled 4-bit matrices from their definition, in numpy with 64 bits: what the GPU tests compare with.  Also the
storage order of fq.h, by its formulas."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FLOOR, COVER = 0, 1


def bf16_values(bits):
    """bf16 bit patterns -> float64."""
    with np.errstate(invalid="ignore"):          # signalling NaNs
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def philox(c, key):
    """Philox4x32-10 of counters c [4, ...] (uint64 arrays of 32-bit values) -> [4, ...]."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) for v in c]
    k0, k1 = key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def random16(rows, cols, seed):
    r, c = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(cols, dtype=np.uint64), indexing="ij")
    zero = np.zeros_like(r)
    words = np.stack(philox([c >> np.uint64(3), r, zero, zero], int(seed)))
    word = np.take_along_axis(words, ((c >> np.uint64(1)) & np.uint64(3)).astype(np.int64)[None], axis=0)[0]
    return ((word >> (np.uint64(16) * (c & np.uint64(1)))) & np.uint64(0xFFFF)).astype(np.int64)


def scale_byte(m, rule):
    """E8M0 byte of a group with largest magnitude m (float64 holding a bf16 value)."""
    if m == 0.0:
        return 0
    e = int(np.frexp(m)[1]) - 1
    s = e - 2
    if rule == COVER and m > 6.0 * 2.0 ** s:
        s += 1
    return max(s, -127) + 127


def quantize(bits, rule=FLOOR, random=None):
    """(E2M1 codes [R, C], scale bytes [R, ceil(C / 32)]) of bf16 bits along the rows; random: 16 random bits per
    element for stochastic rounding (rule COVER then)."""
    x = bf16_values(bits)
    R, Ccols = x.shape
    codes, scales = np.zeros((R, Ccols), np.uint8), np.zeros((R, -(-Ccols // 32)), np.uint8)
    for g in range(scales.shape[1]):
        cut = slice(32 * g, min(32 * g + 32, Ccols))
        v = x[:, cut]
        bad = ~np.isfinite(v).all(axis=1)
        with np.errstate(invalid="ignore"):
            m = np.where(bad, 0.0, np.abs(v).max(axis=1))
        b = np.array([scale_byte(t, rule) for t in m])
        t = np.abs(np.where(bad[:, None], 0.0, v)) / np.ldexp(1.0, b - 127)[:, None]
        lo = np.searchsorted(GRID, t, side="right") - 1
        hi = np.minimum(lo + 1, 7)
        step = np.where(hi > lo, GRID[hi] - GRID[lo], 1.0)
        if random is None:
            f = (t - GRID[lo]) / step
            up = (f > 0.5) | ((f == 0.5) & (lo % 2 == 1))
        else:
            f = (np.floor(t * 2.0 ** 17) / 2.0 ** 17 - GRID[lo]) / step
            up = f + random[:, cut] / 65536.0 >= 1.0
        k = np.where(up & (lo < 7), hi, lo).astype(np.uint8)
        k |= (np.signbit(v).astype(np.uint8) << 3)
        codes[:, cut] = np.where(bad[:, None], 0, k)
        scales[:, g] = np.where(bad, 255, b)
    return codes, scales


def values(codes, scales):
    """What codes and scale bytes stand for, float64 (NaN for byte 255)."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def untile_codes(stored, R, C):
    """[strips, nkb, 1024] bytes -> (codes [R, C], all of the padded codes)."""
    strips, nkb, _ = stored.shape
    r, c = np.meshgrid(np.arange(strips * 16), np.arange(nkb * 128), indexing="ij")
    byte = stored[r // 16, c // 128, (r % 16 + 16 * (c % 128 // 32)) * 16 + c % 32 // 2]
    full = (byte >> (4 * (c % 2)).astype(np.uint8)) & 15
    return full[:R, :C], full


def untile_scales(stored, R, C):
    """[quads, nkb, 256] bytes -> (scales [R, ceil(C / 32)], all of the padded scales)."""
    quads, nkb, _ = stored.shape
    r, g = np.meshgrid(np.arange(quads * 64), np.arange(nkb * 4), indexing="ij")
    full = stored[r // 64, g // 4, (r % 16 + 16 * (g % 4)) * 4 + r // 16 % 4]
    return full[:R, :-(-C // 32)], full
