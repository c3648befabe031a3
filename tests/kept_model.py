"""Pages that hold keys and values in 8 or 4 bits, as wise.h defines them, in
numpy: which code a value becomes, where its byte lies, and back.  Shares no code
with the library.  Values are bf16, given and returned in fp64."""

import numpy as np

TOP = {4: 7.0, 8: 464.0}
RANGE = {4: (-125, 125), 8: (-117, 119)}


def magnitudes(bits):
    """By code; E4M3's last one is NaN."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    out = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(out[:-1] + [np.nan])


def quantise(x, bits):
    """(codes [..., d], scale bytes [..., d / 32]) of x [..., d]: the nearest code."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0, y)
    a = np.abs(y).max(-1)
    lo, hi = RANGE[bits]
    e = np.full(a.shape, lo)
    for k in range(lo + 1, hi + 1):                  # the least e that is enough, or the largest there is
        e = np.where(a > TOP[bits] * 2.0 ** (k - 1), k, e)
    e = np.where(a == 0, 0, e)
    table = magnitudes(bits)[:8 if bits == 4 else 127]
    z = np.abs(y) / 2.0 ** e[..., None].astype(float)
    middle = (table[1:] + table[:-1]) / 2            # between codes i and i + 1; on it, the even one of the two
    low, high = np.searchsorted(middle, z, "left"), np.searchsorted(middle, z, "right")
    codes = np.where(low % 2 == 0, low, high)
    codes = codes | (np.signbit(y).astype(np.int64) << (bits - 1))
    codes = np.where(bad[..., None], 0, codes)
    return codes.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, bits):
    t = magnitudes(bits)
    v = np.concatenate([t, -t])[codes]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(*v.shape[:-1], -1, 32) * s[..., None]).reshape(v.shape)


def page_bytes(page, d, bits):
    return page * (d * bits // 8 + d // 32)


def places(page, d, bits, plane):
    """(byte, shift) of every (token, dim)'s code, and the byte of every (token, scale): read off the definition."""
    row, g = d * bits // 8, d // 32
    code, shift, scale = np.zeros((page, d), int), np.zeros((page, d), int), np.zeros((page, g), int)
    for t in range(page):
        for i in range(d):
            shift[t, i] = 4 * (i % 2) if bits == 4 else 0
            within = i * bits // 8
            if plane == 0:
                code[t, i] = t * row + within
            else:
                sixteenth = d // 16 * bits // 8
                code[t, i] = t // 4 * (4 * row) + i // (d // 16) * (4 * sixteenth) + t % 4 * sixteenth + i % (d // 16) * bits // 8 \
                    if (d // 16 * bits) % 8 == 0 else -1
        for s in range(g):
            scale[t, s] = page * row + (t * g + s if plane == 0 else t // 4 * (4 * g) + 4 * s + t % 4)
    return code, shift, scale


def pack(codes, scales, bits, plane, fill=0):
    """Page bytes [..., page_bytes] of codes [..., page, d] and scales [..., page, d / 32]."""
    page, d = codes.shape[-2:]
    code, shift, scale = places(page, d, bits, plane)
    out = np.zeros((*codes.shape[:-2], page_bytes(page, d, bits)), dtype=np.uint8)
    for half in ((0, 4) if bits == 4 else (0,)):
        m = shift == half
        out[..., code[m]] |= (codes[..., m] << half).astype(np.uint8)
    out[..., scale.reshape(-1)] = scales.reshape(*scales.shape[:-2], -1)
    return out


def unpack(raw, page, d, bits, plane):
    """(codes, scales) of page bytes [..., page_bytes]."""
    code, shift, scale = places(page, d, bits, plane)
    return raw[..., code] >> shift.astype(np.uint8) & (15 if bits == 4 else 255), raw[..., scale]


def read(raw, page, d, bits, plane):
    return values(*unpack(raw, page, d, bits, plane), bits)


def read_pool(pool, page, d, bits):
    """(keys, values) [pages][kv][page][d] of one layer's planes, uint8 [2][pages][kv][page_bytes]."""
    return read(pool[0], page, d, bits, 0), read(pool[1], page, d, bits, 1)


def attend(q, k_pool, v_pool, tables, lens, ids, page, scale):
    """(o, lse, bound, lse_bound) in fp64, as cache_model.attend, with the bounds that 11-bit probabilities allow.

    o is rounded to bf16: half a step, 2^-8 |o|.  A probability enters the product with V in fp16 (or as two bf16 numbers, which
    leaves less): half a step, 2^-12 of it, so 2^-12 A in all, A = sum p |v|; where the row's reference makes it a subnormal, it is off
    by at most 2^-25 while the row's largest is 2^6 or more, which is 2^-31 of z: n 2^-31 max |v|.  A score is an fp32 sum of d exact
    products, off by at most E = scale d 2^-24 max sum |q k| (its own rounding and the scale's, 2^-23 of |s|, in it for d >= 64), which
    changes a probability and the sum by e^E each; the exponentials, and rescaled partial sums over n keys, one
    fp32 rounding of each product's sum: 2^-18 + n 2^-24.  Below fp32's normal numbers a probability, taken against the
    row's largest (so that z >= 1), and either of two parts may become 0: 2^-126 each, 2^-125 sum |v| in all; so may o: 2^-126."""
    batch, heads, q_len, d = q.shape
    pages, kv = k_pool.shape[:2]
    gq = heads // kv
    o, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    bound, lse_bound = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(batch):
        s = ids[b]
        n = min(max(int(lens[s]), 0), tables.shape[1] * page) if 0 <= s < len(lens) else 0
        pos = np.arange(n)
        pg = tables[s][pos // page] if n else np.zeros(0, int)
        ok = (pg >= 0) & (pg < pages)
        for kh in range(kv):
            see = pos[ok]
            k, v = k_pool[pg[see], kh, see % page], v_pool[pg[see], kh, see % page]
            for t in range(q_len):
                m = see <= n - q_len + t
                if not m.any():
                    continue
                kk, vv, hs = k[m], v[m], slice(kh * gq, (kh + 1) * gq)
                qq = q[b, hs, t]
                x = scale * (qq @ kk.T)
                top = x.max(-1, keepdims=True)
                p = np.exp(x - top)
                z = p.sum(-1, keepdims=True)
                p /= z
                o[b, hs, t] = p @ vv
                lse[b, hs, t] = (top + np.log(z))[:, 0]
                e = scale * d * 2.0 ** -24 * (np.abs(qq) @ np.abs(kk).T).max(-1)
                extra = 2.0 ** -12 + 2 * e + 2.0 ** -18 + m.sum() * 2.0 ** -24
                small = m.sum() * 2.0 ** -31 * np.abs(vv).max(0) + 2.0 ** -125 * np.abs(vv).sum(0) + 2.0 ** -126
                bound[b, hs, t] = 2.0 ** -8 * np.abs(o[b, hs, t]) + (1 + 2.0 ** -8) * (extra[:, None] * (p @ np.abs(vv)) + small)
                lse_bound[b, hs, t] = e + 2.0 ** -18 + m.sum() * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse[b, hs, t])
    return o, lse, bound, lse_bound
