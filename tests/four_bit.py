"""Plain definitions, in 64 bits and plain loops or numpy, of what the library does in four bits: the format, the layouts, the
step's plan and the attention.  Shares nothing with the kernels but the documented layout."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """[..., 32] float64 -> (codes, scale bytes): see include/moin.h."""
    x = np.asarray(x, dtype=np.float64)
    broken = ~np.isfinite(x).all(-1)
    v = np.where(broken[..., None], 0.0, x)
    top = np.abs(v).max(-1)
    # the smallest unit in which the largest value rounds to 6 or less (7 would go to 8)
    units = 2.0 ** np.arange(-125, 126)
    e = np.minimum((top[..., None] / units >= 7).sum(-1), 250) - 125
    d = np.abs(np.abs(v)[..., None] / 2.0 ** e[..., None, None] - LEVELS)
    d = np.concatenate([d[..., 0::2], d[..., 1::2]], -1)   # the even codes first: they win ties
    codes = np.array([0, 2, 4, 6, 1, 3, 5, 7], dtype=np.uint8)[d.argmin(-1)] | np.where(v < 0, 8, 0).astype(np.uint8)
    scales = np.where(broken, 255, np.where(top == 0, 127, e + 127)).astype(np.uint8)
    return codes, scales


def level(code):
    return np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7]


def power(E):
    E = np.asarray(E).astype(np.int64)
    return np.where(E == 255, np.nan, np.ldexp(1.0, (E - 127).astype(np.int32)))


def dequantise(codes, scales):
    return level(codes) * power(scales)[..., None]


def held(x):
    """The values that MXFP4 holds for x [..., n], n a multiple of 32."""
    b = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, 32))
    return dequantise(*quantise(b)).reshape(x.shape)


def decode_pages(data, n_pages, n_kv, D, page_tokens):
    """Bytes of a cache -> keys, values [n_pages * page_tokens, n_kv, D] float64, byte by byte as documented."""
    rec = np.asarray(data, dtype=np.uint8).reshape(n_pages, n_kv, page_tokens // 64, 68 * D)
    k = np.empty((n_pages, page_tokens, n_kv, D))
    v = np.empty_like(k)
    ch = np.arange(D)
    for tok in range(page_tokens):
        blk, t = divmod(tok, 64)
        i, m = divmod(t, 16)
        r = rec[:, :, blk]
        kb = r[:, :, i * 8 * D + (ch // 32) * 256 + m * 16 + (ch % 32) // 2]
        vb = r[:, :, 32 * D + i * 8 * D + (ch // 8) * 64 + m * 4 + (ch % 8) // 2]
        ks = r[:, :, 64 * D + (ch // 32) * 64 + m * 4 + i]
        vs = r[:, :, 66 * D + (ch // 32) * 64 + m * 4 + i]
        k[:, tok] = level(kb >> (4 * (ch % 2)) & 15) * power(ks)
        v[:, tok] = level(vb >> (4 * (ch % 2)) & 15) * power(vs)
    return k.reshape(-1, n_kv, D), v.reshape(-1, n_kv, D)


def decode_weight(data, d_out, d_in):
    R, C = -(-d_out // 16), -(-d_in // 512)
    rec = np.asarray(data, dtype=np.uint8).reshape(R, C, 4352)
    W = np.empty((d_out, d_in))
    col = np.arange(d_in)
    j, g, c = col % 512 // 128, col % 128 // 32, col % 32
    for row in range(d_out):
        m = row % 16
        r = rec[row // 16, col // 512]
        at = np.arange(d_in)
        b = r[at, j * 1024 + g * 256 + m * 16 + c // 2]
        W[row] = level(b >> (4 * (c % 2)) & 15) * power(r[at, 4096 + g * 64 + m * 4 + j])
    return W


def plan(kv_lens, new_lens, T, max_new, page, table, free, n_free):
    """(table, kv_lens, seq_offsets, slots, n_free, fault) after a step, request by request."""
    table = [list(map(int, r)) for r in table]
    lens, off, slots, fault = [], [0], [-1] * T, False
    wanted = taken = at = 0
    n_free = int(n_free)
    if n_free < 0 or n_free > len(free):
        fault, n_free = True, min(max(n_free, 0), len(free))
    for s, (kv, n) in enumerate(zip(map(int, kv_lens), map(int, new_lens))):
        sane = kv >= 0 and 0 <= n <= max_new and kv + n <= len(table[s]) * page
        have = -(-max(kv, 0) // page)
        need = -(-(kv + n) // page) - have if sane else 0
        end = at + max(n, 0)
        ok = sane and end <= T and (need == 0 or wanted + need <= n_free)
        fault |= not ok
        if ok:
            for j in range(need):
                table[s][have + j] = int(free[n_free - 1 - (wanted + j)])
            for i in range(n):
                slots[at + i] = table[s][(kv + i) // page] * page + (kv + i) % page
            taken = max(taken, wanted + need) if need else taken
        wanted += need
        lens.append(kv + n if ok else max(kv, 0))
        at = end
        off.append(min(at, T))
    fault |= at != T
    return table, lens, off, slots, n_free - taken, fault


def attention(q, k, v, pos0, scale, window):
    """One request: q [n, heads, D], k / v [L, n_kv, D]; token i at position pos0 + i.  Returns y, lse and, for error
    bounds, sum_j p_j |v_j| and per row the largest relative error of a weight that fp32 scores may cause."""
    n, heads, D = q.shape
    L, n_kv = k.shape[0], k.shape[1]
    y, spread = np.zeros((n, heads, D)), np.zeros((n, heads, D))
    lse, rel = np.full((n, heads), -np.inf), np.zeros((n, heads))
    eps = 2.0 ** -24
    for i in range(n):
        p = pos0 + i
        lo = max(0, p - window + 1) if window else 0
        hi = min(p + 1, L)
        if hi <= lo:
            continue
        for h in range(heads):
            kk, vv = k[lo:hi, h // (heads // n_kv)], v[lo:hi, h // (heads // n_kv)]
            s = scale * (kk @ q[i, h])
            m = s.max()
            w = np.exp(s - m)
            lse[i, h] = m + np.log(w.sum())
            w /= w.sum()
            y[i, h] = w @ vv
            spread[i, h] = w @ np.abs(vv)
            absolute = scale * (np.abs(kk) @ np.abs(q[i, h]))
            # a sum of D products, the scaling, the distance to the maximum, the exponential itself; the sums over the keys
            rel[i, h] = ((D + 2) * eps * absolute + 4 * eps * (np.abs(s) + abs(m))).max() + 2.0 ** -21 + (hi - lo) * eps
    return y, lse, spread, rel
