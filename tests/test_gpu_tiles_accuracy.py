"""How exact slkv_attend_prompt and slkv_attend_tree are on average, against the float64 oracle: limits that a weight held in fewer bits would not keep.  The reasoning is that of
test_gpu_attend_accuracy.py, u = 2^-24: a logit is off by 3.5 u (root mean square), fp32 outputs by 5 u of sum p |v|, the log-sum-exp by 12 u.

16-bit outputs: with values between 1 and 2 whose rounding falls anywhere between two steps, an output that is off by e before it is rounded differs from the rounded exact one with the
probability e / step.  Weights enter the products with V to 2^-16 and a part of 2^-20 of themselves (fp16: towards 0, to 2^-20), so e is at most twice that and 10 u: 2^-15 + 2^-19 + 10 u of a
step of 2^-7, 0.43 %, and 2^-19 + 10 u of a step of 2^-10, 0.26 %.  (One 16-bit number a weight: 5 % and 6 % for 40 rows.)"""

import numpy as np
import pytest
import torch

from oracle import decode
from oracle.prompt import attend_prompt
from paper_2508_15806_amd import api
from decode_parity import DTYPES, cache_values, f64, normal, random_cache
from test_gpu_attend_accuracy import U, positive_values, rms
from test_gpu_prompt import inputs, offsets, values
from test_gpu_tree import random_parents, truth

pytestmark = pytest.mark.gpu


def check(dtype, out, lse, want, want_lse, spread):
    assert rms(f64(lse) - want_lse) <= 12 * U
    if dtype == "f32":
        assert rms((f64(out) - want) / spread) <= 5 * U
        return
    exact = torch.from_numpy(want).to(out.dtype)
    differ = float((out.cpu() != exact).double().mean())
    limit = (2.0 ** -19 + 10 * U) / 2.0 ** -10 if dtype == "f16" else (2.0 ** -15 + 2.0 ** -19 + 10 * U) / 2.0 ** -7
    assert differ <= limit, "%g of the outputs are not the rounded exact ones, %g may" % (differ, limit)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16", "bf16_kv8"])
@pytest.mark.parametrize("Hq,Hkv,n,m", [(16, 4, 1, 40), (32, 4, 7, 40), (16, 4, 3, 3000), (32, 4, 40, 300), (8, 2, 700, 700), (64, 1, 300, 1300)])
def test_prompts(dtype, Hq, Hkv, n, m):
    rng = np.random.default_rng([n, m, Hq])
    cu_q, cu_k = offsets([n]), offsets([m])
    q, k, v = inputs(rng, dtype, Hq, Hkv, 128, cu_q, cu_k)
    if dtype == "bf16_kv8":
        v = torch.from_numpy(rng.integers(0x38, 0x40, tuple(v.shape)).astype(np.uint8)).cuda()
    else:
        v.copy_(torch.from_numpy(rng.uniform(1, 2, tuple(v.shape)).astype(np.float32)))
    out, lse = api.PromptCall(dtype, 1, Hq, Hkv, 128, cu_q, cu_k).run(q, k, v)
    torch.cuda.synchronize()
    want, wl, _, spread = attend_prompt(f64(q), values(k), values(v), cu_q, cu_k)
    # (a query that sees few keys has few weights, each a large share; of those of a whole prompt the first are left out)
    first = min(n - 1, max(0, 40 - (m - n)))
    check(dtype, out[:, first:], lse[:, first:], want[:, first:], wl[:, first:], spread[:, first:])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G,T", [(4, 3), (8, 16), (4, 64)])
@pytest.mark.parametrize("n", [40, 3000])
def test_trees(dtype, G, T, n):
    rng = np.random.default_rng([n, G, T])
    cache = random_cache(rng, dtype, 1, 4, G, 128, [n + T] * 4)
    positive_values(cache, rng)
    q, bits = normal(rng, (1, 4 * G, T, 128), dtype), api.tree_bits(random_parents(rng, 1, T)).cuda()
    out, lse = cache.attend_tree(q, bits)
    torch.cuda.synchronize()
    want, wl, _, spread = decode.attend_tree(f64(q), *cache_values(cache), cache.layout.offsets, [n + T] * 4, 4, truth(bits, T))
    check(dtype, out, lse, want, wl, spread)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv,n,m", [(4, 4, 3, 700), (8, 2, 70, 900), (16, 2, 1000, 1000), (64, 1, 500, 1500)])
@pytest.mark.parametrize("query", [0.0, 1.0])
def test_infinite_values_that_all_see(dtype, Hq, Hkv, n, m, query):
    """A weight times an infinity is one, where the weight is a power of two (equal logits) and where it is not."""
    rng = np.random.default_rng([n, m])
    cu_q, cu_k = offsets([n]), offsets([m])
    q, k, v = inputs(rng, dtype, Hq, Hkv, 128, cu_q, cu_k)
    q *= query
    v[:, 10, 3] = float("inf")
    v[:, 11, 70] = -float("inf")
    v[:, 12, 9], v[:, 200, 9] = float("inf"), -float("inf")
    out, lse = api.PromptCall(dtype, 1, Hq, Hkv, 128, cu_q, cu_k).run(q, k, v)
    torch.cuda.synchronize()
    out, first = out[:, max(0, 201 - (m - n)):], [3, 9, 70]
    assert bool((out[:, :, 3] == float("inf")).all()) and bool((out[:, :, 70] == -float("inf")).all()) and bool(torch.isnan(out[:, :, 9]).all())
    assert bool(torch.isfinite(out[:, :, [c for c in range(128) if c not in first]]).all()) and bool(torch.isfinite(lse).all())
