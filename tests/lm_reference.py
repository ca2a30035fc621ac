"""Plain references of the decoder's operators, in numpy, from their definitions in include/ifq.h."""
import numpy as np

GROUP = 16


def group_bytes(D):
    return 16 * D + 128


def k_place(D):
    """Byte and shift, within a group, of the K code of (row, d): two arrays [16][D]."""
    DB = min(D, 128)
    row, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    # [D / DB][16 tokens][DB] fields of 4 bits
    field = ((d // DB) * 16 + row) * DB + d % DB
    return field // 2, 4 * (field % 2)


def v_place(D):
    """The same for V: [D / DB][2][8][4][DB / 32][2][4], token = 8 a1 + 2 a3 + a5, dimension = DB/8 a2 + 4 a4 + a6."""
    DB = min(D, 128)
    S = DB // 8
    row, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    a0, dd = d // DB, d % DB
    a1, a3, a5 = row // 8, row % 8 // 2, row % 2
    a2, a4, a6 = dd // S, dd % S // 4, dd % 4
    field = (((((a0 * 2 + a1) * 8 + a2) * 4 + a3) * (DB // 32) + a4) * 2 + a5) * 4 + a6
    return 8 * D + field // 2, 4 * (field % 2)


def to_bf16(x):
    """float -> the nearest bfloat16, as float32 (ties to even; finite values)"""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def rotate(x, cos, sin, rope, rot):
    """float32 [T][H][D], tables [T][rot/2], operation by operation"""
    y = x.copy()
    if rope == "none":
        return y
    c, s = cos[:, None].astype(np.float32), sin[:, None].astype(np.float32)
    ia = np.arange(rot // 2) if rope == "halves" else np.arange(0, rot, 2)
    ib = ia + rot // 2 if rope == "halves" else ia + 1
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def quantise4(x):
    """float32 [..., D] -> codes, scale (half), min (half)"""
    with np.errstate(all="ignore"):
        x = np.clip(x.astype(np.float32), np.float32(-65504), np.float32(65504))
        lo, hi = x.min(-1), x.max(-1)
        scale = ((hi - lo) * np.float32(1 / 15)).astype(np.float16)
        mn = lo.astype(np.float16)
        s, m = scale.astype(np.float32)[..., None], mn.astype(np.float32)[..., None]
        code = np.clip(np.rint((x - m) / s), 0, 15)
        code = np.where(s > 0, code, 0)
    return code.astype(np.uint8), scale, mn


def write(cache, page_size, slot, head, D, kq, vq):
    """Put one token's quantised head into cache uint8 [pages][heads][groups][bytes]."""
    page, off = divmod(int(slot), page_size)
    g = cache[page, head, off // GROUP]
    row = off % GROUP
    for (place, (code, scale, mn), at) in ((k_place, kq, 0), (v_place, vq, 64)):
        byte, shift = place(D)
        for d in range(D):
            b, sh = byte[row, d], shift[row, d]
            g[b] = (g[b] & ~(15 << sh) & 255) | (int(code[d]) << sh)
        par = np.array([scale, mn], np.float16).view(np.uint8)
        g[16 * D + at + 4 * row:16 * D + at + 4 * row + 4] = par


def read(cache, page_size, slots, D):
    """float64 values (k, v) [T][heads][D] of the slots (float32 arithmetic is exact to one rounding here)"""
    page, off = np.asarray(slots) // page_size, np.asarray(slots) % page_size
    g = cache[page, :, off // GROUP]                      # [T][heads][bytes]
    row = off % GROUP
    out = []
    for place, at in ((k_place, 0), (v_place, 64)):
        byte, shift = place(D)
        idx = np.broadcast_to(byte[row][:, None], (len(row), g.shape[1], D))
        code = (np.take_along_axis(g, idx, 2) >> shift[row][:, None]) & 15
        pi = np.broadcast_to((16 * D + at + 4 * row)[:, None, None] + np.arange(4), (len(row), g.shape[1], 4))
        par = np.ascontiguousarray(np.take_along_axis(g, pi, 2)).view(np.float16)
        with np.errstate(all="ignore"):
            out.append((code * par[..., :1].astype(np.float64) + par[..., 1:].astype(np.float64), code, par))
    return out


def fill(rng, cache, page_size, slots, D, spread=1.0):
    """Fill the given slots with plausible tokens (codes of every value, scales and minima of both signs)."""
    heads = cache.shape[1]
    for slot in np.asarray(slots).reshape(-1):
        page, off = divmod(int(slot), page_size)
        row = off % GROUP
        g = cache[page, :, off // GROUP]
        for place, at in ((k_place, 0), (v_place, 64)):
            byte, shift = place(D)
            code = rng.integers(0, 16, (heads, D)).astype(np.uint8)
            b = byte[row]
            two = code[:, shift[row] == 0] | (code[:, shift[row] == 4] << 4)
            g[:, b[shift[row] == 0]] = two
            scale = rng.uniform(0.05, 0.3, heads) * spread
            par = np.stack([scale, -7.5 * scale + rng.normal(0, 0.2, heads) * spread], -1).astype(np.float16)
            g[:, 16 * D + at + 4 * row:16 * D + at + 4 * row + 4] = par.view(np.uint8).reshape(heads, 4)


def attention(q, cache, page_size, table, lens, starts, kv_heads, scale, window, sinks, u_out, half_values=False):
    """q float64 [T][Hq][D] -> out, lse, and how far a computation in single precision with half-precision weights
    may be off in each (per element of out, per row of lse).

    The bounds: the scores' sums of D products and the two affine terms err by at most (D + 8) 2^-23 of the sum T of
    their absolute values; a relative change of the weights by e^(2 delta) moves the output by 2 delta A, A the sum of
    p_j |V_j| with |V_j| <= s'_j c'_j + |m'_j|; rounding a weight to half moves it by 2^-11, or by 2^-24 of the largest
    weight below the normal range; with half_values each V_j is rounded to half as well (2^-11 of it, or 2^-24); sums of n terms add n 2^-24 at most for each of the two sums; u_out is the result's
    own rounding."""
    T, Hq, D = q.shape
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    tol, ltol = np.zeros((T, Hq, D)), np.zeros((T, Hq))
    G = Hq // kv_heads
    for s in range(len(lens)):
        a, e = int(starts[s]), int(starts[s + 1])
        n, length = e - a, int(lens[s])
        if n == 0 or length == 0:
            continue
        j = np.arange(length)
        slots = table[s, j // page_size].astype(np.int64) * page_size + j % page_size
        (k, kc, kp), (v, vc, vp) = read(cache, page_size, slots, D)
        for h in range(kv_heads):
            kabs = kc[:, h] * np.abs(kp[:, h, :1].astype(np.float64)) + np.abs(kp[:, h, 1:].astype(np.float64))
            vabs = vc[:, h] * np.abs(vp[:, h, :1].astype(np.float64)) + np.abs(vp[:, h, 1:].astype(np.float64))
            for i in range(n):
                p = length - n + i
                see = (j <= p) & ((window == 0) | (j > p - window) | (j < sinks))
                if not see.any():
                    continue
                for g in range(G):
                    x = q[a + i, h * G + g]
                    with np.errstate(all="ignore"):
                        t = (k[see, h] @ x) * scale
                        top = t.max()
                        w = np.exp(t - top)
                        l = w.sum()
                        o = (w @ v[see, h]) / l
                        delta = (D + 8) * 2.0 ** -23 * np.max(kabs[see] @ np.abs(x)) * abs(scale)
                        A = (w @ vabs[see]) / l
                        m = see.sum()
                        vr = 2.0 ** -11 * A + 2.0 ** -24 if half_values else 0.0
                        tol[a + i, h * G + g] = (vr + u_out * np.abs(o) + (2 * delta + 2.0 ** -11 + 2 * m * 2.0 ** -24) * A +
                                                 m * 2.0 ** -24 * vabs[see].max() / l + 1e-30)
                        out[a + i, h * G + g] = o
                        lse[a + i, h * G + g] = top + np.log(l)
                        ltol[a + i, h * G + g] = delta + m * 2.0 ** -24 + 2.0 ** -21 * max(1.0, abs(top + np.log(l)))
    return out, lse, tol, ltol


# ------------------------------------------------------------------------------------ e4m3


def e4m3_table():
    """The value of every byte."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e.astype(np.float64) - 7))
    v = np.where(b & 128, -v, v)
    v[(b & 127) == 127] = np.nan
    return v


def fp8_quantise(x):
    """float32 [M][K] -> bytes [M][K], scales float32 [blocks][M]"""
    M, K = x.shape
    kb = -(-K // 128)
    tab = e4m3_table()[:127]                     # the non-negative finite values, ascending
    mid = (tab[1:] + tab[:-1]) / 2
    out, scales = np.zeros((M, K), np.uint8), np.zeros((kb, M), np.float32)
    for b in range(kb):
        blk = x[:, 128 * b:128 * b + 128].astype(np.float32)
        s = np.abs(blk).max(1) * np.float32(1 / 448)
        scales[b] = s
        with np.errstate(all="ignore"):
            y = np.where(s[:, None] != 0, blk / s[:, None], np.float32(0))
        mag = np.abs(y).astype(np.float64)
        lo = np.searchsorted(mid, mag, side="left")      # ties are settled below
        tie = (lo < len(mid)) & (mag == mid[np.minimum(lo, len(mid) - 1)])
        code = np.where(tie & (lo % 2 == 1), lo + 1, lo)
        out[:, 128 * b:128 * b + 128] = np.minimum(code, 126) | (np.signbit(y).astype(np.uint8) << 7)
    return out, scales


def fp8_matmul(xq, xs, wq, ws):
    """-> product in float64 and the sum of the absolute values of its terms"""
    tab = e4m3_table()
    M, K = xq.shape
    N = wq.shape[0]
    y, mag = np.zeros((M, N)), np.zeros((M, N))
    for b in range(xs.shape[0]):
        c = slice(128 * b, min(128 * b + 128, K))
        f = xs[b][:, None].astype(np.float64) * np.repeat(ws[:, b].astype(np.float64), 128)[:N]
        y += f * (tab[xq[:, c]] @ tab[wq[:, c]].T)
        mag += np.abs(f) * (np.abs(tab[xq[:, c]]) @ np.abs(tab[wq[:, c]]).T)
    return y, mag
