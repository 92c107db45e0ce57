"""How exact slkv_attend_cache is on average, against the float64 oracle: limits that a weight held in fewer bits, or a shorter sum, would not keep.

u = 2^-24.  With queries and keys of unit variance a product q . k is a sum of d = 128 terms in 2 to 4 chains; the partial sum of i terms has a
magnitude of sqrt(i) and adds a rounding of at most u / sqrt(3) of it (root mean square), so a chain of 32 is off by u sqrt(32^2 / 6) = 13 u, four chains by 26 u,
two of 64 by 37 u, and the joining of them and rounded products by some 10 u: at most 39 u / sqrt(128) = 3.5 u of a logit, which is as much of its softmax weight.  (Products of 16-bit
types are exact and 32 of them are one instruction.)

fp32 outputs: a sum of p v is off by at most 3.5 u S, S = sum p |v|, were all weights off the same way; the exponential, the sums, the division: 1.5 u S more.
Weights that the caller gets: exp2 of c q . k - lse, two numbers below 16 in magnitude, each rounded once or twice by at most 8 u: sqrt(3) 8 u / sqrt(3) ln 2 = 5.6 u,
with the logit's 3.5 u less than 7 u; lse itself: 5.6 u and the sum's 1.5 u.  The limits are 5 u for outputs, 12 u for the others.

16-bit outputs: with values between 1 and 2 whose rounding falls anywhere between two steps, an output that is off by e before it is rounded differs from the rounded exact
one with the probability e / step.  Weights enter the products with V to 2^-16 of themselves (fp16: 2^-21), so e is at most twice that and 10 u: 2^-15 + 10 u
of a step of 2^-7, 0.4 %, and 2^-20 + 10 u of a step of 2^-10, 0.16 %.  (One 16-bit number a weight: 5 % and 6 % for 40 rows.)"""

import numpy as np
import pytest
import torch

from oracle import decode
from decode_parity import DTYPES, cache_values, f64, normal, random_cache

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


def positive_values(cache, rng):
    """V between 1 and 2."""
    rows = cache.rows_in_all
    if cache.dtype == "bf16_kv4":                        # 1 and 1.5
        cache.v_scale.fill_(127)
        cache.v.copy_(torch.from_numpy(rng.choice(np.array([0x22, 0x23, 0x32, 0x33], dtype=np.uint8), (rows, cache.d // 2))))
    elif cache.dtype == "bf16_kv8":
        cache.v.copy_(torch.from_numpy(rng.integers(0x38, 0x40, (rows, cache.d)).astype(np.uint8)))
    else:
        cache.v.copy_(torch.from_numpy(rng.uniform(1, 2, (rows, cache.d)).astype(np.float32)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G,T", [(4, 1), (8, 4), (16, 4)])
@pytest.mark.parametrize("n", [40, 3000])
def test_outputs(dtype, G, T, n):
    rng = np.random.default_rng([n, G, T, DTYPES.index(dtype)])
    cache = random_cache(rng, dtype, 1, 4, G, 128, [n] * 4)
    positive_values(cache, rng)
    q = normal(rng, (1, 4 * G, T, 128), dtype)
    out, lse = cache.attend(q, weight=False)
    want, wl, _, _, spread = decode.attend(f64(q), *cache_values(cache), cache.layout.offsets, [n] * 4, 4, T)
    assert rms(f64(lse) - wl) <= 12 * U
    if dtype == "f32":
        assert rms((f64(out) - want) / spread) <= 5 * U
        return
    exact = torch.from_numpy(want).to(out.dtype)
    differ = float((out.cpu() != exact).double().mean())
    limit = (2.0 ** -20 + 10 * U) / 2.0 ** -10 if dtype == "f16" else (2.0 ** -15 + 10 * U) / 2.0 ** -7
    assert differ <= limit, "%g of the outputs are not the rounded exact ones, %g may" % (differ, limit)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [40, 3000])
def test_weights(dtype, n):
    """One query a segment: what it adds to a row is the row's softmax weight."""
    rng = np.random.default_rng([n, DTYPES.index(dtype)])
    cache = random_cache(rng, dtype, 8, 4, 1, 128, [n] * 32)
    cache.weight.zero_()
    q = normal(rng, (8, 4, 1, 128), dtype)
    cache.attend(q)
    want = decode.attend(f64(q), *cache_values(cache), cache.layout.offsets, [n] * 32, 4, 1)[2]
    assert rms((f64(cache.weight) - want) / want) <= 12 * U


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("n", [50, 5000])
def test_logits_at_the_end_of_the_range(dtype, sign, n):
    """Some rows share the largest logit, 2^22 in magnitude; the others are 2^14 and more below: the mean of their values, whatever the logit."""
    rng = np.random.default_rng(n)
    d = 64
    cache = random_cache(rng, dtype, 1, 2, 2, d, [n, n])
    k = np.zeros((2 * n, d), np.float32)
    k[:, 0] = sign * 2.0 ** 13 - (32 + 32 * rng.integers(0, 60, 2 * n))
    for s in range(2):
        k[s * n + rng.permutation(n)[:3], 0] = sign * 2.0 ** 13
    cache.k.copy_(torch.from_numpy(k))                   # (bf16 has steps of 64 above 2^13: more than three rows then)
    q = torch.zeros((1, 4, 1, d), dtype=cache.query_dtype, device="cuda")
    q[..., 0] = 2.0 ** 12                                # x = 2^25 / 8
    cache.weight.zero_()
    out, lse = cache.attend(q)
    held, v, w = f64(cache.k)[:, 0], f64(cache.v), f64(cache.weight)
    half = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    for s in range(2):
        top = s * n + np.flatnonzero(held[s * n:(s + 1) * n] == sign * 2.0 ** 13)
        want = v[top].mean(0)
        # equal weights, which carry the same rounding of the logit; fp32 adds the values and divides
        assert (np.abs(f64(out)[0, 2 * s:2 * s + 2, 0] - want) <= (2.0 ** -15 if half else (5 + len(top)) * U) * np.abs(v[top]).max() + half * np.abs(want)).all()
        assert (np.abs(f64(lse)[0, 2 * s:2 * s + 2, 0] - (sign * 2.0 ** 22 + np.log(len(top)))) <= 0.5).all()
        # 2 queries a segment; exp2 of a difference that is off by the roundings of lse: three numbers below 2^23, half a step of 1/4 each at most
        assert (np.abs(np.log2(w[top] / (2 / len(top)))) <= 0.75).all()
        w[top] = 0
    assert (w == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "bf16_kv4"])
@pytest.mark.parametrize("n", [33, 6000])
def test_values_at_the_end_of_the_range(dtype, n):
    """Values of one sign and 2^118 over the rows: their mean, though their sum comes near the largest number."""
    rng = np.random.default_rng(n)
    cache = random_cache(rng, dtype, 1, 2, 4, 64, [n, n])
    e = 118 - int(np.ceil(np.log2(n)))
    if dtype == "bf16_kv4":
        cache.v_scale.fill_(127 + e)
        cache.v.fill_(0x22)
    else:
        cache.v.fill_(2.0 ** e)
    q = normal(rng, (1, 8, 1, 64), dtype) * 3
    out, _ = cache.attend(q)
    assert (np.abs(f64(out) / 2.0 ** e - 1) <= 2.0 ** -15 + (2.0 ** -20 + 16 * U if dtype == "f32" else 2.0 ** -8)).all()
