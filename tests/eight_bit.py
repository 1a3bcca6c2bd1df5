"""Plain definitions, in 64 bits and plain loops or numpy, of what the library does in eight bits: E4M3, the cache's blocks and their
scales, the rotation, the integer product.  Shares nothing with the kernels but the documented layouts."""
import numpy as np

LD = np.longdouble


# ---- E4M3 -------------------------------------------------------------------------------------------------

def e4m3_values():
    """What the 256 codes stand for."""
    c = np.arange(256)
    e, m = c >> 3 & 15, (c & 7).astype(np.float64)
    mag = np.where(e == 0, m * 2.0 ** -9, np.ldexp(8 + m, e - 10))
    mag[(c & 127) == 127] = np.nan
    return np.where(c > 127, -mag, mag)


VALUES = e4m3_values()


def e4m3(x):
    """Codes of x (float64), nearest, ties to even, magnitudes above 448 clamped."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    e = np.maximum(np.frexp(a)[1] - 1, -6)
    n = np.rint(np.ldexp(a, 3 - e)).astype(np.int64)          # in units of the last place: 0 .. 16
    code = np.where(n < 8, n, (e + 7) * 8 + n - 8)            # (n = 16 carries into the exponent)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_byte(top):
    """E of values whose largest magnitude is `top` (NaN or infinity among them: not finite)."""
    if not np.isfinite(top):
        return 255
    for e in range(-117, 119):
        if top < 464.0 * 2.0 ** e:
            return e + 127
    return 246


def power(E):
    return np.nan if E == 255 else float(np.ldexp(1.0, int(E) - 127))


# ---- the cache ----------------------------------------------------------------------------------------------

class Cache:
    """Bytes of a paged cache, block by block as documented."""

    def __init__(self, data, n_pages, n_kv, D, page):
        self.data = np.array(data, dtype=np.uint8).reshape(n_pages, -1)
        self.n_kv, self.D, self.page, self.B = n_kv, D, page, page // 64
        t, c = np.arange(64)[:, None], np.arange(D)[None]
        self.k_at = t // 16 * 16 * D + c // 64 * 1024 + t % 16 * 64 + c % 64
        self.v_at = 64 * D + c // 16 * 1024 + c % 16 * 64 + t // 4 % 4 * 16 + t // 16 * 4 + t % 4

    def places(self, page, head, blk, is_v):
        """Byte of each [token, channel] of a block, and of its scale, in the page."""
        at = (head * self.B + blk) * 128 * self.D
        return at + (self.v_at if is_v else self.k_at), self.n_kv * self.B * 128 * self.D + 2 * (head * self.B + blk) + is_v

    def append(self, k, v, off, slots):
        for s in range(len(off) - 1):
            mine = [int(x) for x in slots[off[s]:off[s + 1]]]
            i = 0
            while i < len(mine) and mine[0] != -1:
                n = min(len(mine) - i, 64 - mine[i] % 64)
                page, blk, p0 = mine[i] // self.page, mine[i] % self.page // 64, mine[i] % 64
                for h in range(self.n_kv):
                    for is_v, x in enumerate((k, v)):
                        self.block(page, h, blk, is_v, p0, np.asarray(x[off[s] + i:off[s] + i + n, h], dtype=np.float64))
                i += n

    def block(self, page, h, blk, is_v, p0, x):
        at, sc = self.places(page, h, blk, is_v)
        row = self.data[page]
        E0 = int(row[sc]) if p0 else 0
        E1 = scale_byte(np.abs(x).max())
        E = max(E0, E1)
        if E0 and E > E0 and E != 255:
            row[at[:p0]] = e4m3(VALUES[row[at[:p0]]] * 2.0 ** (E0 - E))
        row[sc] = E
        if E != 255:
            row[at[p0:p0 + len(x)]] = e4m3(x / power(E))

    def values(self):
        """Keys and values [n_pages * page, n_kv, D] that the bytes stand for."""
        n = self.data.shape[0]
        out = np.empty((2, n, self.B, 64, self.n_kv, self.D))
        with np.errstate(invalid="ignore", over="ignore"):
            for h in range(self.n_kv):
                for b in range(self.B):
                    for is_v in range(2):
                        at, sc = self.places(0, h, b, is_v)
                        E = self.data[:, sc]
                        unit = np.where(E == 255, np.nan, np.ldexp(1.0, E.astype(np.int32) - 127))
                        out[is_v, :, b, :, h] = VALUES[self.data[:, at]] * unit[:, None, None]
        return out.reshape(2, -1, self.n_kv, self.D)


# ---- norms and rotation ---------------------------------------------------------------------------------------

def norm_rope(x, pos, freqs, gain, eps, norm, neighbours):
    """x [T, heads, D] -> (result, magnitude that the rotation's errors are relative to), float64."""
    x = np.asarray(x, dtype=np.float64)
    if norm:
        with np.errstate(invalid="ignore", over="ignore"):
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if gain is not None:
            x = x * gain
    out, size = x.copy(), np.abs(x)
    if pos is not None:
        n = len(freqs)
        angle = np.fmod(np.asarray(pos).astype(LD)[:, None] * np.asarray(freqs).astype(LD), 2 * np.arccos(LD(-1)))
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if neighbours else (slice(0, n), slice(n, 2 * n))
        a, b = x[..., i], x[..., j]
        out[..., i], out[..., j] = a * c - b * s, b * c + a * s
        size[..., i] = size[..., j] = np.abs(a) + np.abs(b)
    return out, size


# ---- integers ---------------------------------------------------------------------------------------------------

def integers(x):
    """Rows of x -> (codes, scales): see include/moin.h."""
    x = np.asarray(x, dtype=np.float64)
    top = np.abs(x).max(1)
    bad = ~np.isfinite(top)
    s = np.maximum((np.where(bad, 1.0, top) / 127.0).astype(np.float32), np.float32(2.0 ** -126)).astype(np.float64)
    # the quotient's fraction decides exactly: x has 8 bits, s 24, and 64 bits hold their products
    q = np.rint(np.where(bad[:, None], 0.0, x) / s[:, None])
    left = np.where(bad[:, None], 0.0, x) - q * s[:, None]
    q += np.where(np.abs(left) > s[:, None] / 2, np.sign(left), 0)
    return q.astype(np.int64), np.where(bad, np.nan, s)
