"""A cache of 8- or 4-bit elements: 32 neighbours share a power of two.

Everything by search over the format's list of values: no bit tricks, float64.  Test infrastructure only.
"""
import numpy as np

BLOCK, PAGE, LEAST = 32, 64, -100


def _magnitudes(fmt):
    """The magnitudes of the format in code order."""
    if fmt == "e2m1":
        return np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    v = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(v[:-1])                                # (the last code is NaN)


def quantise(x, fmt):
    """x [..., D] -> (codes uint8 [..., D], one element each; scale bytes uint8 [..., D / 32])."""
    x = np.asarray(x, np.float64)
    mags = _magnitudes(fmt)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK, BLOCK))
    flat = b.reshape(x.size // BLOCK, BLOCK)
    finite = np.isfinite(flat).all(axis=1)
    flat = np.where(finite[:, None], flat, 0.0)
    top, e = np.abs(flat).max(axis=1, initial=0.0), np.full(len(flat), float(LEAST))
    while (over := top > mags[-1] * 2.0 ** e).any():
        e[over] += 1
    y = np.abs(flat) / 2.0 ** e[:, None]
    hi = np.searchsorted(mags, y).clip(0, len(mags) - 1)
    lo = (hi - 1).clip(0)
    d_hi, d_lo = np.abs(mags[hi] - y), np.abs(y - mags[lo])
    pick = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    codes = (pick + (len(mags) + (fmt == "e4m3")) * np.signbit(flat)).astype(np.uint8)
    codes[~finite] = 0
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    return codes.reshape(x.shape), scales.reshape(b.shape[:-1])


def values(codes, scales, fmt):
    """What codes [..., D] (one element each) and scale bytes stand for, float64."""
    mags = _magnitudes(fmt)
    n = 128 if fmt == "e4m3" else 8
    table = np.concatenate([mags, [np.nan] * (n - len(mags)), -mags, [np.nan] * (n - len(mags))])
    v = table[np.asarray(codes, np.int64)]
    s = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales, np.float64) - 127))
    return (v.reshape(v.shape[:-1] + (-1, BLOCK)) * s[..., None]).reshape(v.shape)


def store(k, rows_of, lens, table, n_pages, codes, scales, fmt):
    """Rows of k join a cache in place: rows_of[s] lists the rows that sequence s stores behind its lens[s] tokens; codes
    [n_pages, Hkv, 64, D] (one element each), scales [n_pages, Hkv, 64, D / 32].  Returns the lengths afterwards."""
    new = np.array(lens, np.int64)
    k_codes, k_scales = quantise(k, fmt)
    for s, rows in enumerate(rows_of):
        for r in rows:
            t = int(new[s])
            if t >= len(table[s]) * PAGE:
                break
            new[s] += 1
            page = int(table[s][t // PAGE])
            if 0 <= page < n_pages:
                codes[page, :, t % PAGE], scales[page, :, t % PAGE] = k_codes[r], k_scales[r]
    return new


def fetch(codes, scales, table, s, tokens, fmt):
    """Values [tokens, Hkv, D] of the given tokens of sequence s."""
    out = [values(codes[int(table[s][t // PAGE]), :, t % PAGE], scales[int(table[s][t // PAGE]), :, t % PAGE], fmt) for t in tokens]
    return np.stack(out) if out else np.zeros((0, codes.shape[1], codes.shape[3]))
