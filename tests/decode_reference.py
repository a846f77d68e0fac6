"""The operators around decoding from their definitions, in 64 bits with NumPy, and how far a kernel may be from them."""
import numpy as np


def rope(x, positions, inv_freq, interleaved=False, magnitude=1.0, inverse=False):
    x = np.asarray(x, np.float64)
    rot = 2 * len(inv_freq)
    a = np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64)
    c, s = np.cos(a)[:, None] * magnitude, np.sin(a)[:, None] * magnitude * (-1 if inverse else 1)
    y = x.copy()
    i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., i] * s + x[..., j] * c
    return y


def quantize(x, bits):
    """(codes, fp32 scales) of the vectors along the last axis."""
    x = np.asarray(x, np.float64)
    top = 127 if bits == 8 else 7
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0, x)
    scale = (np.abs(x).max(-1) / top).astype(np.float32)
    codes = np.where(scale[..., None] > 0, np.rint(x / np.where(scale > 0, scale, 1).astype(np.float64)[..., None]), 0)
    return np.clip(codes, -top, top).astype(np.int8), np.where(bad, np.float32(np.nan), scale)


def unpack(codes, bits):
    """Codes as int8, from the cache's bytes."""
    codes = np.asarray(codes)
    if bits == 8:
        return codes
    c = codes.view(np.int8)
    return np.stack([(c << 4).astype(np.int8) >> 4, c >> 4], -1).reshape(*c.shape[:-1], -1)


def pack(codes, bits):
    return codes if bits == 8 else ((codes[..., 0::2] & 15) | (codes[..., 1::2] << 4)).astype(np.uint8)


def attention(q, kc, vc, ks, vs, table, lengths, starts, tree=None, scale=None, half_step=2.0 ** -24, weight_step=2.0 ** -20, own_exponents=True):
    """(result, tolerance) of one call; rows of no sequence are NaN.  kc, vc: int8 codes (pages, heads, page, dk).

    Tolerance of a row with weights p, values v and result o, A = sum p |v|:
      half_step |o|       the result's rounding
      weight_step A       each weight's rounding for the second product
      A (e^(2 d) - 1)     scores off by d: q c is summed over dk elements in fp32 (dk + 8 roundings of the sum of |q c|, 2^-24 each), and
                          q is held to 2^-22 of the row's largest at worst
      (keys + 16) 2^-23 A sums over the keys, the exponentials and the rescalings
      2^-29 w sum |c|     weights are halves, or sums of two, times a power of two such that the row's largest p 2^e, e the exponent of V's scale, lies between 2^7 and 2^15 (it is
                          brought to 2^7 when it is beyond 2^15).  A half's step is never below 2^-24, so each of up to two halves is off by up to 2^-25, a weight by 2^-31 of that
                          largest, and p 2^e is up to four times w, the largest p times scale: of one token (own_exponents), or, where several tokens share the
                          exponent of their largest scale, of any two of them
    """
    q = np.asarray(q, np.float64)
    pages, kv_heads, page, dk = kc.shape
    group = q.shape[1] // kv_heads
    scale = 1 / np.sqrt(dk) if scale is None else scale
    out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b, length in enumerate(lengths):
        s0, s1 = int(starts[b]), int(starts[b + 1])
        n, length = s1 - s0, int(min(max(length, 0), table.shape[1] * page))
        t = np.arange(length)
        ids = table[b, t // page].astype(np.int64)
        good = (ids >= 0) & (ids < pages)
        ids = np.where(good, ids, 0)
        later = t - (length - n)
        for i in range(n):
            if tree is None:
                seen = later <= i
            else:
                seen = (later < 0) | ((later >= 0) & (np.uint64(tree[s0 + i]) >> np.clip(later, 0, 63).astype(np.uint64) & np.uint64(1)).astype(bool))
            at = np.nonzero(seen & good)[0]
            for h in range(q.shape[1]):
                out[s0 + i, h], tol[s0 + i, h] = 0, 0
                if len(at) == 0:
                    continue
                kh = h // group
                kcode, vcode = kc[ids[at], kh, at % page].astype(np.float64), vc[ids[at], kh, at % page].astype(np.float64)
                k_s, v_s = ks[ids[at], kh, at % page].astype(np.float64), vs[ids[at], kh, at % page].astype(np.float64)
                row = q[s0 + i, h]
                x = (kcode @ row) * k_s * scale
                e = np.exp(x - x.max())
                p = e / e.sum()
                v = vcode * v_s[:, None]
                o = p @ v
                spread = p @ np.abs(v)
                d = (((np.abs(kcode) @ np.abs(row)) * (dk + 8) * 2.0 ** -24 + np.abs(kcode).sum(1) * np.abs(row).max() * 2.0 ** -22) * k_s * abs(scale)).max()
                out[s0 + i, h] = o
                largest = (p * np.abs(v_s)).max() if own_exponents else p.max() * np.abs(v_s).max()
                tol[s0 + i, h] = 2.0 ** -29 * largest * np.abs(vcode).sum(0) + half_step * np.abs(o) + spread * (weight_step + np.expm1(2 * d) + (len(at) + 16) * 2.0 ** -23) + 1e-30
    return out, tol
