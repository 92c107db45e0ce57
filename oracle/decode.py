"""Decoding on a compacted cache, in float64, from the definitions: 8- and 4-bit values, attention over the rows in use with the weight that each
row gets, eviction by accumulated weight.  One loop per segment, nothing shared with the kernels."""

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127])
BLOCK = 32


def _nearest(mag, grid):
    """Codes of the nearest grid values, ties to the even code, beyond the last one the last."""
    mag = np.minimum(mag, grid[-1])
    hi = np.clip(np.searchsorted(grid, mag, side="left"), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = mag - grid[lo], grid[hi] - mag
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def to_e4m3(x):
    """float64 values -> E4M3 bytes: finite values saturate at 448, infinities and NaN become NaN."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x)
    code = _nearest(np.where(bad, 0, np.abs(x)), E4M3) | (np.signbit(x).astype(np.int64) << 7)
    return np.where(bad, (np.signbit(x).astype(np.int64) << 7) | 0x7F, code).astype(np.uint8)


def from_e4m3(b):
    mag = np.append(E4M3, np.nan)[b & 127]
    return np.where(b & 128, -mag, mag)


def block_exponents(x):
    """Exponents [.., d/32] of x [.., d]: the smallest integer e >= -127 with max |block| <= 7 * 2^e; None's place, 128, for a block that is not finite."""
    b = np.abs(np.asarray(x, np.float64)).reshape(x.shape[:-1] + (-1, BLOCK))
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0, b.max(-1))
    e = np.full(top.shape, -127)
    for k in range(-126, 128):
        e = np.where(top > 7 * 2.0 ** (k - 1), k, e)
    return np.where(bad, 128, e)


def to_mxfp4(x):
    """[.., d] float64 -> (bytes [.., d/2], exponent bytes [.., d/32])."""
    x = np.asarray(x, np.float64)
    e = block_exponents(x)
    b = x.reshape(x.shape[:-1] + (-1, BLOCK))
    with np.errstate(invalid="ignore"):
        mag = np.where(e[..., None] == 128, 0, np.abs(b) / 2.0 ** np.minimum(e, 127)[..., None])
    code = (_nearest(mag, E2M1) | (np.signbit(b).astype(np.int64) << 3)).reshape(x.shape)
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8), (e + 127).astype(np.uint8)


def from_mxfp4(codes, exps):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(c & 8, -E2M1[c & 7], E2M1[c & 7]).reshape(c.shape[:-1] + (-1, BLOCK))
    scale = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return (v * scale[..., None]).reshape(c.shape)


def attend(q, k, v, offsets, lengths, Hkv, T, weight=None):
    """q [B][Hq][T][d]; k, v [rows][d] float64 values; segment s = b*Hkv + h uses rows offsets[s] .. + lengths[s].  Returns out [B][Hq][T][d],
    lse [B][Hq][T], weight [rows] (given or zeros, plus this call's), and what a result's error is measured by: per query the
    largest sum of |q_i k_i| / sqrt(d) over its rows, per (query, dim) the weighted sum of |v|."""
    q = np.asarray(q, np.float64)
    B, Hq, _, d = q.shape
    G = Hq // Hkv
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    weight = np.zeros(k.shape[0]) if weight is None else np.array(weight, np.float64)
    terms, spread = np.zeros(q.shape[:3]), np.zeros(q.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(B):
            for hq in range(Hq):
                s = b * Hkv + hq // G
                a, n = int(offsets[s]), int(lengths[s])
                for t in range(T):
                    m = n - T + 1 + t
                    if m <= 0:
                        continue
                    kk, vv = k[a:a + m], v[a:a + m]
                    x = (kk * q[b, hq, t]).sum(1) / np.sqrt(d)
                    top = x.max()
                    p = np.exp(x - top)
                    lse[b, hq, t] = top + np.log(p.sum())
                    p = p / p.sum()
                    out[b, hq, t] = (p[:, None] * vv).sum(0)
                    weight[a:a + m] += p
                    t_all = np.abs(kk) @ np.abs(q[b, hq, t])           # (a logit that is not finite carries no rounding)
                    terms[b, hq, t] = t_all[np.isfinite(t_all)].max(initial=0.0) / np.sqrt(d)
                    spread[b, hq, t] = p @ np.abs(vv)
    return out, lse, weight, terms, spread


def evict_segment(weight, w, cap):
    """Row numbers that stay of a segment with these weights: the max(cap, w) - w largest of all but the last w (equal ones: the lower row; NaN
    above all numbers), ascending, then the last w."""
    n, room = len(weight), max(cap, w)
    if n <= room:
        return np.arange(n)
    m = n - w
    rank = sorted(range(m), key=lambda j: (0 if np.isnan(weight[j]) else 1, 0.0 if np.isnan(weight[j]) else -float(weight[j]), j))
    return np.array(sorted(rank[:room - w]) + list(range(m, n)), dtype=np.int64)
