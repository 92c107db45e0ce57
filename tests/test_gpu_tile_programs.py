"""Every program of the attention of prompts and of drafted trees (tile_cases.py) against the float64 oracle, some heads of each."""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2508_15806_amd import api
from decode_parity import cache_values, f64, normal, random_cache
from test_gpu_prompt import check, inputs, offsets
from test_gpu_tree import random_parents, truth
from tile_cases import PROMPTS, TREES
from tile_parity import check_outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,waves,kind,Hq,Hkv,n,m", PROMPTS)
def test_prompts(dtype, d, waves, kind, Hq, Hkv, n, m):
    rng = np.random.default_rng([Hq, Hkv, sum(n)])
    cu_q, cu_k = offsets(n, 3), offsets(n if m is None else m, 2)
    q, k, v = inputs(rng, dtype, Hq, Hkv, d, cu_q, cu_k)
    out, lse = api.PromptCall(dtype, len(n), Hq, Hkv, d, cu_q, cu_k).run(q, k, v)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for h in sorted({0, Hkv // 2, Hkv - 1}):
        heads = sorted({h * G, h * G + G // 2, h * G + G - 1})
        check(dtype, len(heads), 1, d, cu_q, cu_k, q[heads], k[h:h + 1], v[h:h + 1], out[heads], lse[heads])


@pytest.mark.parametrize("dtype,d,waves,kind,Hq,Hkv,seqs,T,room", TREES)
def test_trees(dtype, d, waves, kind, Hq, Hkv, seqs, T, room):
    rng = np.random.default_rng([Hq, Hkv, T, room])
    S, G = seqs * Hkv, Hq // Hkv
    lens = [room - int(rng.integers(0, max(1, room // 6))) for _ in range(S)]
    lens[0], lens[S // 2] = room, min(room, T // 2)          # a full room; a draft that is not all there
    cache = random_cache(rng, dtype, seqs, Hkv, G, d, lens, rooms=[room] * S)
    q, bits = normal(rng, (seqs, Hq, T, d), dtype), api.tree_bits(random_parents(rng, seqs, T)).cuda()
    out, lse = cache.attend_tree(q, bits)
    torch.cuda.synchronize()
    k, v = cache_values(cache)
    for s in sorted({0, S // 2, S - 1}):
        b, h = divmod(s, Hkv)
        rows, heads = slice(s * room, (s + 1) * room), sorted({h * G, h * G + G - 1})
        o, l, terms, spread = decode.attend_tree(f64(q[b:b + 1, heads]), k[rows], v[rows], [0, room], lens[s:s + 1], 1, truth(bits[b:b + 1], T))
        check_outputs(dtype, d, room, out[b:b + 1, heads], lse[b:b + 1, heads], o, l, terms, spread, np.abs(v[rows][np.isfinite(v[rows])]).max(initial=0.0))
