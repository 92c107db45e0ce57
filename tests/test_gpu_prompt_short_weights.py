"""slkv_attend_prompt with SLKV_PROMPT_SHORT_WEIGHTS: one number a weight, because the caller says so.  Logits, softmax and log-sum-exp are those of the other calls, bit for bit; outputs are within the
roundings that tile_parity.py counts, half a step of the queries' type a weight among them."""

import numpy as np
import pytest
import torch

from paper_2508_15806_amd import api
from decode_parity import f64
from test_gpu_prompt import check, inputs, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16", "bf16_kv8"])
@pytest.mark.parametrize("Hq,Hkv,d,n,m", [(8, 2, 128, [1, 2, 40], [300, 1000, 40]), (4, 2, 64, [65, 0, 300], [70, 5, 290]), (32, 8, 128, [700, 40], None), (64, 8, 64, [800], None),
                                          (64, 1, 128, [600, 0, 500, 30], [600, 4, 900, 20]), (8, 2, 128, [500], [9000]), (256, 8, 128, [205, 0, 42, 39, 120, 366], [205, 4, 32, 39, 120, 368])])
def test_against_the_oracle(dtype, Hq, Hkv, d, n, m):
    rng = np.random.default_rng([Hq, d, sum(n)])
    cu_q, cu_k = offsets(n, 1), offsets(n if m is None else m, 2)
    q, k, v = inputs(rng, dtype, Hq, Hkv, d, cu_q, cu_k)
    want, lse2 = api.PromptCall(dtype, len(n), Hq, Hkv, d, cu_q, cu_k).run(q, k, v)
    out, lse = api.PromptCall(dtype, len(n), Hq, Hkv, d, cu_q, cu_k, short_weights=True).run(q, k, v)
    torch.cuda.synchronize()
    a = int(cu_q[0])
    assert torch.equal(lse[:, a:], lse2[:, a:]) and (dtype != "f32" or torch.equal(out[:, a:], want[:, a:]))
    G = Hq // Hkv
    for h in sorted({0, Hkv - 1}):
        heads = sorted({h * G, h * G + G - 1})
        check(dtype, len(heads), 1, d, cu_q, cu_k, q[heads], k[h:h + 1], v[h:h + 1], out[heads], lse[heads])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinite_values(dtype):
    rng = np.random.default_rng(3)
    cu = offsets([600])
    q, k, v = inputs(rng, dtype, 4, 2, 128, cu, cu)
    v[:, 10, 3], v[:, 450, 5] = float("inf"), float("nan")
    out, _ = api.PromptCall(dtype, 1, 4, 2, 128, cu, short_weights=True).run(q, k, v)
    torch.cuda.synchronize()
    assert bool((out[:, 10:, 3] == float("inf")).all()) and bool(torch.isfinite(out[:, :10]).all()) and bool(torch.isfinite(out[:, :450, 5]).all()) and bool(torch.isnan(out[:, 450:, 5]).all())
    assert bool(torch.isfinite(out[..., [c for c in range(128) if c not in (3, 5)]]).all())


def test_the_choice_is_a_captured_calls_too():
    rng = np.random.default_rng(4)
    cu_q, cu_k = offsets([4, 30]), offsets([5000, 3001])
    q, k, v = inputs(rng, "bf16", 8, 2, 128, cu_q, cu_k)
    calls = [api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k, short_weights=short) for short in (False, True)]
    want = [[x.clone() for x in c.run(q, k, v)] for c in calls]
    assert not torch.equal(want[0][0], want[1][0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = [c.run(q, k, v) for c in calls]
    for _ in range(3):
        for x in got:
            x[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
        assert np.isfinite(f64(got[1][0])).all()
