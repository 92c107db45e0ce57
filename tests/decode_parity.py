"""What the tests of the calls on a cache share: random caches, their values in float64, and how far results may be off.

Tolerances count roundings.  With u = 2^-24: a logit is a sum of d exact products in fp32, off by at most d u times the largest sum of
magnitudes `terms` (queries and keys of E4M3, MXFP4, bf16 and fp16 have exact products; fp32 ones add d u of their own) and, scaled by a rounded constant
and turned into a power of two by the chip, by 4 u of itself and 2^-22 of the result: e = (2 d + 8) u terms + 2^-21, the logits' magnitude being at
most `terms`.  A softmax weight is off by at most 2 e of itself and the rounding of a sum of n terms (blocks of at most n / 16 + 64 in a
row): r = 2 e + (n / 16 + 64) u.  Weights go into the products with V to 2^-16 of themselves.  So with S = sum p |v| an output is off by (r + 2^-15) S and the
rounding to its own type, half a step."""

import numpy as np
import torch

from oracle import decode
from paper_2508_15806_amd import api

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11, "bf16_kv8": 2.0 ** -8, "bf16_kv4": 2.0 ** -8}
DTYPES = ["f32", "bf16", "f16", "bf16_kv8", "bf16_kv4"]


def normal(rng, shape, dtype):
    """A device tensor in the type of the queries."""
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(api.CACHE_DTYPES[dtype][1]).cuda()


def f64(t):
    return t.double().cpu().numpy()


def cache_values(cache):
    """K and V of every row as float64."""
    def values(x, e):
        if cache.dtype == "bf16_kv4":
            return decode.from_mxfp4(x.cpu().numpy(), e.cpu().numpy())
        return decode.from_e4m3(x.cpu().numpy()) if cache.dtype == "bf16_kv8" else f64(x)
    return values(cache.k, cache.k_scale), values(cache.v, cache.v_scale)


def random_cache(rng, dtype, B, Hkv, G, d, lens, rooms=None, before=0, fill=float("nan")):
    """A Cache with lens[s] random rows in use; the rows behind them (and before the first room) hold `fill` in K and V."""
    rooms = lens if rooms is None else rooms
    offsets = np.concatenate([[0], np.cumsum(rooms)]).astype(np.int64) + before
    cache = api.Cache(dtype, B, Hkv * G, Hkv, d, offsets)
    rows = int(offsets[-1])
    # through the oracle's own narrowing: the kernels that narrow have tests of their own
    for x, e in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        vals = normal(rng, (rows, d), dtype)
        used = np.zeros(rows, bool)
        for s, n in enumerate(lens):
            used[offsets[s]:offsets[s] + n] = True
        unused = torch.from_numpy(~used).cuda()
        vals[unused] = fill
        if dtype == "bf16_kv4":
            codes, exps = decode.to_mxfp4(f64(vals))
            x.copy_(torch.from_numpy(codes))
            e.copy_(torch.from_numpy(exps))
        else:
            x.copy_(torch.from_numpy(decode.to_e4m3(f64(vals))) if dtype == "bf16_kv8" else vals)
    cache.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    cache.weight.copy_(torch.from_numpy(rng.random(rows, dtype=np.float32)))
    cache.pos.copy_(torch.arange(rows, dtype=torch.int32) * 7 + 3)
    return cache


def close(got, want, tol, what):
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(tol, np.shape(want))
    same = np.isnan(want) == np.isnan(got)
    assert same.all(), "%s: NaN in other places: %s" % (what, np.argwhere(~same)[:4])
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), "%s: infinities" % what
    fine = np.isfinite(want)
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    assert off.size == 0 or off.max() <= 0, "%s: off by %g more than %g at %s" % (what, off.max(), tol[fine][off.argmax()], np.argwhere(fine)[off.argmax()])


def check_attend(cache, q, T, out, lse, weight_before=None, weight_after=None, lens=None):
    """Results of one call against the oracle."""
    offsets = cache.layout.offsets
    lens = cache.lengths.cpu().numpy() if lens is None else lens
    k, v = cache_values(cache)
    before = None if weight_before is None else f64(weight_before)
    o, l, w, terms, spread = decode.attend(f64(q), k, v, offsets, lens, cache.Hkv, T, before)
    u, d, n = 2.0 ** -24, cache.d, max([1] + [int(x) for x in lens])
    e = (2 * d + 8) * u * terms + 2.0 ** -21
    r = 2 * e + (n / 16 + 64) * u
    close(f64(out), o, (r[..., None] + 2.0 ** -15) * spread + HALF_STEP[cache.dtype] * np.abs(o), "out")
    close(f64(lse), l, r + 2.0 ** -22 * np.abs(np.where(np.isfinite(l), l, 0)), "lse")
    if weight_after is not None:
        # each of a segment's R queries adds a weight that is off by r of itself; the sum and the addition round
        R = cache.Hq // cache.Hkv * T
        S = len(lens)
        tol = np.zeros_like(w)
        for s in range(S):
            a, m = int(offsets[s]), int(lens[s])
            b, h = divmod(s, cache.Hkv)
            G = cache.Hq // cache.Hkv
            rr = r[b, h * G:(h + 1) * G].max()
            added = w[a:a + m] - (before[a:a + m] if before is not None else 0)
            tol[a:a + m] = (rr + R * u) * np.abs(added) + 2 * u * np.abs(w[a:a + m])
        close(f64(weight_after), w, tol, "weight")
