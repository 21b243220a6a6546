"""The paged cache operators in float64 (numpy), slot by slot from their definition, and
the bounds on what the library's results may be off."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = {"f32": 2.0**-24, "bf16": 2.0**-8, "f16": 2.0**-11}


def to_mxfp4(x):
    """x [..., d] -> the values its codes stand for (blocks of 32 channels)."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    amax = np.abs(b).max(-1, keepdims=True)
    fine = np.isfinite(amax)
    safe = np.where(fine & (amax > 0), amax, 1.0)
    e = np.where(fine & (amax > 0), np.clip(np.frexp(safe)[1] - 3, -127, 127), -127)  # floor(log2 amax) - 2
    y = np.minimum(np.abs(np.where(fine, b, 0.0)) / 2.0**e, 6.0)
    off = np.abs(y[..., None] - GRID)
    even_first = [0, 2, 4, 6, 1, 3, 5, 7]  # argmin takes the first of two equally near: the even code
    code = np.array(even_first)[np.argmin(off[..., even_first], -1)]
    out = np.where(fine, np.copysign(GRID[code] * 2.0**e, b), np.nan)
    return out.reshape(x.shape)


def rotate(x, pos, base):
    """x [rows, heads, d] at pos [rows] with the float32 table's cosines and sines."""
    d = x.shape[-1]
    ang = np.asarray(pos, np.float64)[:, None] * float(np.float32(base)) ** (-2.0 * np.arange(d // 2) / d)
    c, s = (np.asarray(f(ang), np.float32).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    a, b = x[..., 0::2].astype(np.float64), x[..., 1::2].astype(np.float64)
    return np.stack([a * c - b * s, a * s + b * c], -1).reshape(x.shape)


def attend(q, k, v, lo, hi, scale, have=None):
    """q [rows, H, d] of one sequence over k, v [slots, Hk, d]; have [slots]: slots with a
    page.  Returns (out, bound terms): sum p |v|, largest score error per unit of relative
    query error and per unit of absolute query error, largest score, slots seen, sum |v| / l."""
    rows, H, d = q.shape
    n, Hk = k.shape[:2]
    out = np.zeros((rows, H, d))
    pv, rel, ab, top, seen, av = (np.zeros((rows, H, 1)) for _ in range(6))
    pv = np.zeros((rows, H, d))
    av = np.zeros((rows, H, d))
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    for r in range(rows):
        s = np.arange(max(int(lo[r]), 0), min(int(hi[r]), n))
        if have is not None:
            s = s[have[s]]
        if len(s) == 0:
            continue
        for h in range(H):
            kk, vv = k[s, h * Hk // H], v[s, h * Hk // H]
            score = kk @ q[r, h] * scale
            p = np.exp(score - score.max())
            total = p.sum()
            p /= total
            out[r, h] = p @ vv
            pv[r, h] = p @ np.abs(vv)
            av[r, h] = np.abs(vv).sum(0) / total
            rel[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
            ab[r, h] = np.abs(kk).sum(1).max() * np.abs(q[r, h]).max() * abs(scale)
            top[r, h] = np.abs(score).max()
            seen[r, h] = len(s)
    return out, (pv, rel, ab, top, seen, av)


def attend_bound(terms, out, cache, qt, d):
    """Elementwise bound on an attention output's error.  A score is off by what its query
    terms lose (float16 pairs hold a row scaled to its largest value to 2^-22 of it,
    bfloat16 terms 2^-8 of the rest each, equal types nothing) plus the float32 sum over
    the channels and the rounding of the exponent's argument; a probability's relative
    error is twice the largest score error (its own and the sum's), plus the rounding of
    its one to three 16-bit terms and of exp2 (2^-22); the sum over n slots adds n 2^-24."""
    pv, rel, ab, top, seen, av = terms
    same = qt == cache or (cache == "mxfp4" and qt == "bf16")
    f16 = cache == "f16"
    if same or (cache == "mxfp4" and qt == "f16"):
        dq = 0.0
    elif f16:
        dq = 2.0**-22 * ab
    else:
        dq = 2.0**-24 * rel
    ds = dq + (d + 4) * 2.0**-24 * rel + 16 * 2.0**-24 * top
    one = same
    dp = (2.0**-11 if one else 2.0**-22) if f16 else (2.0**-8 if one else 2.0**-16 if qt == "f16" else 2.0**-24)
    lost = 2.0**-24 * av if f16 else 0.0  # probabilities below float16's range
    least = 2.0**-25 if qt == "f16" else 1e-37  # half of the smallest step that the output's type has
    return pv * (2 * ds + dp + 2.0**-21 + (seen + 64) * 2.0**-24) + lost + np.abs(out) * HALF_STEP[qt] * 1.01 + least
