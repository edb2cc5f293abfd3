"""The 4-bit key-value cache and attention over it, in float64, token by token.

Written from the format's definition: one token's bytes are placed and found by
their offsets, with none of the library's tiling.
"""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x float64 [..., d]: codes (0 .. 15) [..., d] and exponent bytes [..., d / 32]."""
    u = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(u).max(-1)
    bad = ~np.isfinite(u).all(-1)
    top = np.where(bad, 0.0, top)
    m, e = np.frexp(top)  # top = m 2^e, m in [.5, 1)
    e = np.where(m >= 0.875, e, e - 1) - 2  # the power's exponent
    # from 2^-127 to 2^125, whose multiples by 6 are still finite in fp32
    byte = np.where(top > 0, np.clip(e + 127, 0, 252), 0)
    y = np.abs(np.where(bad[..., None], 0.0, u)) / 2.0 ** (byte[..., None] - 127.0)
    y = np.minimum(y, 6.0)
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    y = np.rint(y / step) * step  # to nearest even multiple of the step
    code = np.abs(y[..., None] - LEVELS).argmin(-1) + 8 * np.signbit(u)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def values(code, byte):
    v = np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
    return v * np.repeat(s, 32, axis=-1)


def page_bytes(page, H, d):
    return H * (page // 32) * 34 * d


def places(page, d, h, t):
    """Byte offsets of token t (< page) of head h in its page: K codes [d / 2], V codes
    [d / 2], K exponents [d / 32], V exponents [d / 32]."""
    base = (h * (page // 32) + t // 32) * 34 * d
    t %= 32
    b, c, i = t // 16, t % 4, (t // 4) % 4  # t = 16 b + 4 i + c
    blk, byte = np.divmod(np.arange(d // 2), 16)
    k = base + blk * 512 + t * 16 + byte
    v = base + 16 * d + blk * 512 + byte * 32 + i * 8 + b * 4 + c
    x = np.arange(d // 32)
    ke = base + 32 * d + (t % 16) * (d // 16) + 2 * x + b
    ve = base + 33 * d + i * (d // 4) + x * 8 + b * 4 + c
    return k, v, ke, ve


def write(data, page, k, v, slot_page, slot_token):
    """Rows k, v float64 [n, H, d] into data [n_pages, page_bytes] (uint8, in place) at
    (page, token); rows whose page is out of range are dropped."""
    n, H, d = k.shape
    (kc, ke), (vc, ve) = quantise(k), quantise(v)
    for r in range(n):
        p = slot_page[r]
        if p < 0 or p >= data.shape[0]:
            continue
        for h in range(H):
            a, b, c, e = places(page, d, h, int(slot_token[r]))
            data[p, a] = kc[r, h, 0::2] | kc[r, h, 1::2] << 4
            data[p, b] = vc[r, h, 0::2] | vc[r, h, 1::2] << 4
            data[p, c], data[p, e] = ke[r, h], ve[r, h]


def read(data, page, H, d, slot_page, slot_token):
    """(k, v) float64 [n, H, d]; zeros where the page is out of range."""
    n = len(slot_page)
    out = np.zeros((2, n, H, d))
    for r in range(n):
        p = slot_page[r]
        if p < 0 or p >= data.shape[0]:
            continue
        for h in range(H):
            a, b, c, e = places(page, d, h, int(slot_token[r]))
            for w, (code, byte) in enumerate(((a, c), (b, e))):
                x = data[p, code]
                out[w, r, h] = values(np.stack([x & 15, x >> 4], -1).reshape(-1), data[p, byte])
    return out[0], out[1]


def attend(q, k, v, there, length, causal, scale):
    """One sequence: q float64 [n, Hq, d], k and v [tokens >= length, H, d], there [tokens]
    (whether a token's page is in the table).  O [n, Hq, d], LSE [n, Hq], and what bounds
    are made of: the weights' sum of |v| per element, the largest sum of |q k| of a seen key."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    O, LSE = np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf)
    absv, big = np.zeros((n, Hq, d)), np.zeros((n, Hq))
    for i in range(n):
        last = min(length, length - n + i + 1) if causal else length
        seen = np.nonzero(there[:max(last, 0)])[0]
        if seen.size == 0:
            continue
        for h in range(Hq):
            kk, vv = k[seen, h // G], v[seen, h // G]
            s = kk @ q[i, h] * scale
            m = s.max()
            w = np.exp(s - m)
            LSE[i, h] = m + np.log(w.sum())
            w /= w.sum()
            O[i, h] = w @ vv
            absv[i, h] = w @ np.abs(vv)
            big[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return O, LSE, absv, big
