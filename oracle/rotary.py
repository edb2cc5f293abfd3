"""Rotary positions with several axes, in extended precision (numpy longdouble).

Angles are position times frequency with 64 bits of mantissa, so that a
position of 2^31 still has its angle to 1e-9 radians.
"""
import numpy as np


def axes_of(sections, dealt):
    """(axis, index within the axis) of every pair."""
    if not dealt:
        return [(a, j) for a, n in enumerate(sections) for j in range(n)]
    left, out = list(sections), []
    while any(left):
        for a in range(len(sections)):
            if left[a]:
                out.append((a, sections[a] - left[a]))
                left[a] -= 1
    return out


def rotate(x, pos, sections, theta=10000.0, pairs="half", spectrum="shared", dealt=False,
           pos_scale=None, inverse=False):
    """x float64 [B, L, H, d], pos integer [axes, B, L]; the turned x in float64, and
    |a| + |b| of each element's pair (0 where nothing turns)."""
    n = sum(sections)
    y, size = x.astype(np.float64).copy(), np.zeros_like(x, dtype=np.float64)
    for i, (a, j) in enumerate(axes_of(sections, dealt)):
        at = np.longdouble(i) / n if spectrum == "shared" else np.longdouble(j) / sections[a]
        f = np.power(np.longdouble(theta), -at) * (1.0 if pos_scale is None else pos_scale[a])
        w = pos[a].astype(np.longdouble) * f
        w = -w if inverse else w
        c, s = np.cos(w).astype(np.float64)[..., None], np.sin(w).astype(np.float64)[..., None]
        p, q = (i, i + n) if pairs == "half" else (2 * i, 2 * i + 1)
        u, v = x[..., p].astype(np.float64), x[..., q].astype(np.float64)
        y[..., p], y[..., q] = u * c - v * s, v * c + u * s
        size[..., p] = size[..., q] = np.abs(u) + np.abs(v)
    return y, size
