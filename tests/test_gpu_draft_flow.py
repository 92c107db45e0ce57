"""A prompt's attention, its compression, and decoding by drafted trees on what it leaves, until the cache is evicted: the calls in turn, as a program makes them."""

import numpy as np
import pytest
import torch

import oracle
from oracle import decode
from oracle.prompt import attend_prompt
from paper_2508_15806_amd import api
from decode_parity import cache_values, check_attend, f64, normal
from test_gpu_tree import check as check_tree
from tile_parity import check_outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8", "bf16_kv4"])
def test_prompt_compression_drafts_eviction(kind):
    rng = np.random.default_rng(21)
    Bn, Hq, Hkv, d, w, T = 2, 8, 2, 128, 16, 7
    n = [700, 250]
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    q, k, v = (normal(rng, (h, int(cu[-1]), d), "bf16") for h in (Hq, Hkv, Hkv))
    out, lse = api.PromptCall("bf16", Bn, Hq, Hkv, d, cu).run(q, k, v)
    torch.cuda.synchronize()
    check_outputs("bf16", d, max(n), out, lse, *attend_prompt(f64(q), f64(k), f64(v), cu, cu))

    budgets = np.array([60, 200], dtype=np.int32)
    call = api.LayerCall("bf16", Bn, Hq, Hkv, d, w, cu, budgets)
    qwin = torch.stack([q[:, cu[b + 1] - w:cu[b + 1]] for b in range(Bn)])
    call.run(qwin, k, v)
    torch.cuda.synchronize()
    as_bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    ref = oracle.compress_layer(as_bits(qwin), as_bits(k), as_bits(v), cu, budgets, w, 7)
    assert np.array_equal(call.kept_idx.cpu().numpy(), np.concatenate([s["kept_idx"] for s in ref["segments"]]))

    rooms = np.array(call.offsets) + 40 * np.arange(Bn * Hkv + 1)
    cache = api.Cache(kind, Bn, Hq, Hkv, d, rooms)
    cache.fill(call.k_out, call.v_out, call.offsets, call.kept_idx)
    lens = np.diff(call.offsets)
    where = np.array(n)
    parents = np.array([[-1, 0, 0, 1, 1, 2, 4], [-1, 0, 1, 1, 0, 4, 5]])
    bits, path = api.tree_bits(parents).cuda(), np.array([[0, 1, 4, 6], [0, 4, -1, -1]])
    for turn in range(3):
        kn, vn, qn = (normal(rng, (Bn, h, T, d), kind) for h in (Hkv, Hkv, Hq))
        depth = [[0, 1, 1, 2, 2, 2, 3], [0, 1, 2, 2, 1, 2, 3]]
        cache.append(kn, vn, torch.tensor([[int(where[b]) + x for x in depth[b]] for b in range(Bn)], dtype=torch.int32).cuda())
        out, lse = check_tree(cache, qn, bits)
        before = cache.weight.clone()
        cache.accept(torch.from_numpy(path.astype(np.int32)).cuda(), T, q=qn, lse=lse)
        torch.cuda.synchronize()
        count = (path >= 0).sum(1)
        lens = lens + np.repeat(count, Hkv)
        assert cache.lengths.tolist() == lens.tolist()
        for s in range(Bn * Hkv):
            a, c, b = int(rooms[s]), int(count[s // Hkv]), s // Hkv
            m = int(lens[s])
            assert cache.pos[a + m - c:a + m].tolist() == [int(where[b]) + i for i in range(c)]
            # every accepted query has given a weight of 1
            assert abs(float((cache.weight[a:a + m].double().sum() - before[a:a + m - c].double().sum())) - c * Hq // Hkv) < 1e-3
        where = where + count
    # a token as usual
    qn = normal(rng, (Bn, Hq, 1, d), kind)
    cache.append(normal(rng, (Bn, Hkv, 1, d), kind), normal(rng, (Bn, Hkv, 1, d), kind), torch.from_numpy(where[:, None].astype(np.int32)).cuda())
    lens = lens + 1
    before = cache.weight.clone()
    out, lse = cache.attend(qn)
    torch.cuda.synchronize()
    used = torch.zeros_like(before, dtype=torch.bool)
    for s, m in enumerate(lens):
        used[int(rooms[s]):int(rooms[s]) + int(m)] = True
    check_attend(cache, qn, 1, out, lse, before, torch.where(used, cache.weight, before))
    small = api.Cache(kind, Bn, Hq, Hkv, d, np.concatenate([[0], np.cumsum(np.minimum(np.diff(rooms), np.tile([50, 100], Bn)))]))
    cache.evict([50, 100], 8, small)
    torch.cuda.synchronize()
    weight, pos, k_all = f64(cache.weight), cache.pos.cpu().numpy(), cache_values(cache)[0]
    for s, m in enumerate(lens):
        stay = decode.evict_segment(weight[int(rooms[s]):int(rooms[s]) + int(m)], 8, [50, 100][s % Hkv]) + int(rooms[s])
        a = int(small.layout.offsets[s])
        assert small.lengths[s].item() == len(stay) and small.pos[a:a + len(stay)].tolist() == pos[stay].tolist()
        np.testing.assert_array_equal(cache_values(small)[0][a:a + len(stay)], k_all[stay])
