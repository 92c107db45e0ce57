"""CPU-only tests of slkv_attend_prompt: descriptors, refusals before any GPU call, workspace sizes, the checks of api.PromptCall."""

import contextlib
import ctypes as C
import gc
import types
import weakref

import numpy as np
import pytest
import torch

from oracle.prompt import attend_prompt
from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B

FAKE, ODD, NULL = 4096, 4100, None
BIG = 1 << 50


def batch(strides=None, **over):
    p = dict(dtype=B.SLKV_BF16, B=2, Hq=8, Hkv=2, d=128, cu_q=[0, 30, 50], cu_k=[0, 100, 130])
    p.update(over)
    x = B.PromptBatch(**p)
    x.desc.strides[:] = [128, 50 * 128, 128, 130 * 128, 128, 130 * 128, 128, max(50, int(x.cu_q[-1])) * 128]
    for i, s in (strides or {}).items():
        x.desc.strides[i] = s
    return x


def attend(x=None, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=NULL, ws=FAKE, nbytes=BIG):
    x = x or batch()
    return B.lib().slkv_attend_prompt(x.address, q, k, v, out, lse, ws, nbytes, None)


def test_struct_size_matches_the_header():
    assert C.sizeof(B.PromptDesc) == 8 * 4 + 2 * 8 + 8 * 8


@pytest.mark.parametrize("over,status", [
    (dict(d=96), 4), (dict(Hq=7), 2), (dict(dtype=5), 2), (dict(dtype=-1), 2), (dict(dtype=B.SLKV_BF16_KV_MXFP4), 4), (dict(B=0, cu_q=[0], cu_k=None), 2),
    (dict(cu_q=[0, 30, 20]), 2), (dict(cu_q=[-1, 30, 50]), 2), (dict(cu_k=[0, 100, 90]), 2), (dict(cu_k=[-2, 100, 130]), 2), (dict(cu_q=[0, 1, 2 ** 31]), 2),
    (dict(cu_k=[0, 1, 2 ** 31]), 2), (dict(Hkv=0, Hq=0), 2), (dict(Hq=1 << 17, Hkv=1), 2), (dict(cu_q=[0, 0, 2 ** 30], cu_k=None), 4), (dict(cu_k=[0, 1, 2 ** 30 + 2]), 4),
    (dict(strides={0: 4}), 2), (dict(strides={3: -128}), 2), (dict(strides={2: 1 << 23}), 4), (dict(strides={4: 1 << 23}), 4), (dict(strides={5: 1 << 41}), 2), (dict(strides={0: 1 << 38}), 2), (dict(strides={3: 1 << 39}), 2),
    (dict(strides={6: 0}), 2), (dict(strides={7: 128}), 2), (dict(strides={6: 64}), 2), (dict(strides={7: 49 * 128}), 2), (dict(strides={6: 7 * 128, 7: 128}), 2),
])
def test_refused_descriptors(over, status):
    x = batch(**over)
    with pytest.raises(B.SlkvError) as e:
        B.slkv_prompt_workspace_bytes(x)
    assert e.value.status == status and B.lib().slkv_last_error() != b""
    assert attend(x) == status


def test_descriptor_struct():
    L, n = B.lib(), C.c_size_t(0)
    for change in (dict(struct_size=8), dict(reserved=(C.c_int32 * 2)(0, 1)), dict(h_cu_q=None)):
        x = batch()
        for name, v in change.items():
            setattr(x.desc, name, v)
        assert L.slkv_prompt_workspace_bytes(x.address, C.addressof(n)) in (1, 2) and attend(x) in (1, 2)
    assert L.slkv_prompt_workspace_bytes(None, C.addressof(n)) == 1 and L.slkv_prompt_workspace_bytes(batch().address, None) == 1


def test_options():
    lay = dict(dtype=B.SLKV_BF16, B=2, Hq=8, Hkv=2, d=128, cu_q=[0, 1, 2], cu_k=[0, 9000, 18000])
    plain, short = B.PromptBatch(**lay), B.PromptBatch(options=B.SLKV_PROMPT_SHORT_WEIGHTS, **lay)
    assert B.slkv_prompt_workspace_bytes(plain) == B.slkv_prompt_workspace_bytes(short)
    assert api.PromptCall("bf16", 2, 8, 2, 128, [0, 1, 2], device="cpu:0").batch.desc.reserved[0] == 0
    assert api.PromptCall("bf16", 2, 8, 2, 128, [0, 1, 2], device="cpu:0", short_weights=True).batch.desc.reserved[0] == B.SLKV_PROMPT_SHORT_WEIGHTS
    for bad in (2, 3, -1, 1 << 30):
        x = batch()
        x.desc.reserved[0] = bad
        assert attend(x) == 2


def test_refused_calls():
    for name in ("q", "k", "v", "out", "ws"):
        assert attend(**{name: NULL}) == 1
        assert attend(**{name: ODD}) == 2
    assert attend(lse=ODD) == 2
    x = batch(cu_q=[0, 1, 2], cu_k=[0, 9000, 18000])
    assert attend(x, nbytes=B.slkv_prompt_workspace_bytes(x) - 1) == 5


def test_strides_that_are_allowed():
    for strides in ({6: 128, 7: 50 * 128}, {6: 8 * 128, 7: 128}, {6: 9 * 144, 7: 144}, {0: 0, 1: 0, 2: 0, 3: 0, 4: 0, 5: 0}):
        assert B.slkv_prompt_workspace_bytes(batch(strides=strides)) >= 16
    # (one token, one head: whatever the stride)
    assert B.slkv_prompt_workspace_bytes(batch(B=1, Hq=1, Hkv=1, cu_q=[0, 1], cu_k=None, strides={6: 0, 7: 0})) >= 16


def test_workspace_holds_the_parts_of_few_queries_alone():
    few = B.slkv_prompt_workspace_bytes(batch(cu_q=[0, 1, 2], cu_k=[0, 100000, 200000]))
    many = B.slkv_prompt_workspace_bytes(batch(Hq=32, Hkv=8, cu_q=[0, 30000, 60000], cu_k=None))
    assert few > 4096 and many == 16


def test_prompt_call_checks_its_tensors(monkeypatch):
    call = api.PromptCall("bf16", 2, 8, 2, 128, [0, 30, 50], [0, 100, 130], device="cpu:0")
    call.device = torch.device("cpu")
    monkeypatch.setattr(call, "_on", lambda stream: pytest.fail("the call went through"), raising=False)
    q, k = torch.zeros((8, 50, 128), dtype=torch.bfloat16), torch.zeros((2, 130, 128), dtype=torch.bfloat16)
    for bad in ((q[:, :49], k, k), (q[:7], k, k), (q, k[:, :129], k), (q, k, k[:1]), (q.half(), k, k), (q, k, k.float()), (q[..., :64], k, k),
                (torch.zeros((8, 50, 256), dtype=torch.bfloat16)[..., ::2], k, k), (q, k.view(torch.uint8)[..., :128], k)):
        with pytest.raises(ValueError):
            call.run(*bad)
    with pytest.raises(ValueError):
        api.PromptCall("bf16", 2, 8, 2, 128, [0, 30], device="cpu:0")
    with pytest.raises(ValueError, match="stream"):
        api.PromptCall("bf16", 1, 8, 2, 128, [0, 30], device="cuda:0")._on(types.SimpleNamespace(device=torch.device("cuda", 1)))


def test_prompt_call_keeps_no_outputs(monkeypatch):
    """An output is the caller's alone: its memory, or that of the graph whose capture made it, is free when the caller lets it go."""
    call = api.PromptCall("bf16", 2, 8, 2, 128, [0, 30, 50], device="cpu:0")
    call.device = torch.device("cpu")
    monkeypatch.setattr(call, "_on", lambda stream: contextlib.nullcontext(), raising=False)
    monkeypatch.setattr(B, "_stream", lambda stream: 0)
    monkeypatch.setattr(B, "slkv_attend_prompt", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    q, k = torch.zeros((8, 50, 128), dtype=torch.bfloat16), torch.zeros((2, 50, 128), dtype=torch.bfloat16)
    for _ in range(2):
        kept = [weakref.ref(x) for x in call.run(q, k, k)]
        gc.collect()
        assert all(x() is None for x in kept)


def test_oracle_against_a_loop():
    rng = np.random.default_rng(1)
    cu_q, cu_k = np.array([1, 4, 4, 9]), np.array([0, 2, 7, 20])
    q, k, v = rng.standard_normal((4, 9, 8)), rng.standard_normal((2, 20, 8)), rng.standard_normal((2, 20, 8))
    out, lse, _, _ = attend_prompt(q, k, v, cu_q, cu_k)
    for b in range(3):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        for h in range(4):
            for i in range(n):
                x = [q[h, cu_q[b] + i] @ k[h // 2, cu_k[b] + j] / 8 ** 0.5 for j in range(m) if j <= m - n + i]
                if not x:
                    assert (out[h, cu_q[b] + i] == 0).all() and lse[h, cu_q[b] + i] == -np.inf
                    continue
                p = np.exp(x)
                np.testing.assert_allclose(lse[h, cu_q[b] + i], np.log(p.sum()), rtol=1e-12)
                np.testing.assert_allclose(out[h, cu_q[b] + i], p @ v[h // 2, cu_k[b]:cu_k[b] + len(x)] / p.sum(), rtol=1e-10, atol=1e-14)
