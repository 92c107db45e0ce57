"""The calls together, as a decoding program makes them: a compressed prefill enters the cache, tokens are appended and attend, rows with little weight leave, and
the cache goes back to the selection by pooled importance.  The oracle follows on the host from the same inputs."""

import numpy as np
import pytest
import torch

import oracle
from oracle import decode
from paper_2508_15806_amd import api
from paper_2508_15806_amd import workloads as wl
from decode_parity import DTYPES, cache_values, check_attend, f64, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("graph", [False, True])
def test_prefill_decode_evict_recompress(dtype, graph):
    B_, Hq, Hkv, d, w = 2, 8, 2, 64, 16
    rng = np.random.default_rng(21)
    source = "f32" if dtype == "f32" else "f16" if dtype == "f16" else "bf16"
    lay = wl.make_layer((31,), [900, 300], Hq, Hkv, d, w, dtype=source, bias_frac=0.05)
    bud = np.array([120, 60], dtype=np.int32)
    call = api.LayerCall(source, B_, Hq, Hkv, d, w, lay.cu_seqlens, bud)
    call.run(*(api.to_device(x, source) for x in (lay.qwin, lay.k, lay.v)))
    kept = call.offsets
    room = 24
    rooms = np.concatenate([[0], np.cumsum(np.diff(kept) + room)])
    cache = api.Cache(dtype, B_, Hq, Hkv, d, rooms)
    cache.fill(call.k_out, call.v_out, kept, call.kept_idx)
    assert cache.lengths.cpu().tolist() == np.diff(kept).tolist()
    k, v = normal(rng, (B_, Hkv, 1, d), dtype), normal(rng, (B_, Hkv, 1, d), dtype)
    q, pos = normal(rng, (B_, Hq, 1, d), dtype), torch.zeros((B_, 1), dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((B_, Hq, 1), device="cuda")

    def step():
        cache.append(k, v, pos)
        cache.attend(q, out=out, lse=lse)
    if graph:
        before = [t.clone() for t in (cache.lengths, cache.weight)]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()                                        # allocates the workspace
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
        for t, x in zip((cache.lengths, cache.weight), before):
            t.copy_(x)
    lens = np.diff(kept).copy()
    for i in range(room):
        for t in (k, v, q):
            t.copy_(normal(rng, t.shape, dtype))
        pos.copy_(torch.tensor([[900 + i], [300 + i]], dtype=torch.int32))
        weight_before = cache.weight.clone()
        torch.cuda.synchronize()
        g.replay() if graph else step()
        torch.cuda.synchronize()
        for s in range(B_ * Hkv):
            weight_before[int(rooms[s]) + int(lens[s])] = 0.0
        lens += 1
        assert cache.lengths.cpu().tolist() == lens.tolist()
        used = torch.zeros_like(weight_before, dtype=torch.bool)
        for s in range(B_ * Hkv):
            used[int(rooms[s]):int(rooms[s]) + int(lens[s])] = True
        check_attend(cache, q, 1, out, lse, weight_before, torch.where(used, cache.weight, weight_before))
    # every query gives out one unit of weight
    total = [float(cache.weight[int(rooms[s]):int(rooms[s]) + int(lens[s])].double().sum()) for s in range(B_ * Hkv)]
    assert np.allclose(total, room * Hq // Hkv, rtol=1e-4)

    # eviction back to the capacities, the latest 4 rows safe
    out_rooms = np.concatenate([[0], np.cumsum([max(int(c), 4) for _ in range(B_) for c in bud])])
    small = api.Cache(dtype, B_, Hq, Hkv, d, out_rooms)
    cache.evict(bud, 4, small)
    torch.cuda.synchronize()
    weight, positions = cache.weight.cpu().numpy(), cache.pos.cpu().numpy()
    kv = cache_values(cache), cache_values(small)
    for s in range(B_ * Hkv):
        a, o = int(rooms[s]), int(out_rooms[s])
        stay = decode.evict_segment(weight[a:a + lens[s]], 4, int(bud[s % Hkv])) + a
        n = len(stay)
        assert int(small.lengths[s]) == n
        for full, part in zip(kv[0], kv[1]):
            assert np.array_equal(full[stay], part[o:o + n])
        assert np.array_equal(positions[stay], small.pos[o:o + n].cpu().numpy()) and positions[stay][-1] == [900, 300][s // Hkv] + room - 1
        assert np.array_equal(weight[stay], small.weight[o:o + n].cpu().numpy())

    # and by pooled importance, from the rows as 16-bit values
    counts = small.lengths.cpu().numpy()
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    k_rows, v_rows, p_rows = small.rows(offs)
    tight = np.array([50, 30], dtype=np.int32)
    again = api.RaggedCall(source, B_, Hq, Hkv, d, w, offs, tight)
    qwin = normal(rng, (B_, Hq, w, d), source)
    again.run(qwin, k_rows, v_rows, p_rows)
    torch.cuda.synchronize()
    ref = oracle.recompress_layer(api.to_host(qwin), api.to_host(k_rows), api.to_host(v_rows), offs, tight, w, 7, pos_in=p_rows.cpu().numpy())
    assert np.array_equal(again.kept_idx.cpu().numpy(), np.concatenate([x["kept_idx"] for x in ref["segments"]]))
    assert np.array_equal(again.pos_out.cpu().numpy(), ref["pos_out"])
