"""Causal attention of packed prompts in float64, from the definition.  One loop per sequence and query head, nothing shared with the kernels."""

import numpy as np


def attend_prompt(q, k, v, cu_q, cu_k):
    """q [Hq][queries][d]; k, v [Hkv][tokens][d] float64 values; sequence b has the queries cu_q[b]..cu_q[b+1], those of the latest of its tokens
    cu_k[b]..cu_k[b+1].  Returns out [Hq][queries][d], lse [Hq][queries], and what a result's error is measured by: per query the largest sum
    of |q_i k_i| / sqrt(d) over the keys it sees, per (query, dim) the weighted sum of |v|."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    Hq, _, d = q.shape
    G = Hq // k.shape[0]
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    terms, spread = np.zeros(q.shape[:2]), np.zeros(q.shape)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for b in range(len(cu_q) - 1):
            n, m = int(cu_q[b + 1] - cu_q[b]), int(cu_k[b + 1] - cu_k[b])
            new = slice(int(cu_q[b]), int(cu_q[b + 1]))
            sees = np.arange(m)[None] <= m - n + np.arange(n)[:, None]
            some = sees.any(1)
            if not some.any():
                continue
            for hq in range(Hq):
                kk, vv = k[hq // G, cu_k[b]:cu_k[b + 1]], v[hq // G, cu_k[b]:cu_k[b + 1]]
                qq = q[hq, new]
                x = np.where(sees, qq @ kk.T / np.sqrt(d), -np.inf)
                top = np.where(some, x.max(1, initial=-np.inf), 0.0)[:, None]
                p = np.where(sees, np.exp(x - top), 0.0)
                total = p.sum(1, keepdims=True)
                lse[hq, new] = np.where(some, (top + np.log(total))[:, 0], -np.inf)
                p = p / np.where(some[:, None], total, 1.0)
                clean = np.isfinite(vv)
                o = p @ np.where(clean, vv, 0.0)
                for j, c in np.argwhere(~clean):               # (0 times an infinity would reach queries that do not see it)
                    o[sees[:, j], c] += p[sees[:, j], j] * vv[j, c]
                out[hq, new] = np.where(some[:, None], o, 0.0)
                t_all = np.where(sees, np.abs(qq) @ np.abs(kk).T, 0.0)
                terms[hq, new] = np.where(np.isfinite(t_all), t_all, 0.0).max(1, initial=0.0) / np.sqrt(d)
                spread[hq, new] = np.where(some[:, None], p @ np.abs(np.where(clean, vv, 0.0)), 0.0)
    return out, lse, terms, spread
