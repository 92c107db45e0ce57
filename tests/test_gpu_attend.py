"""slkv_attend_cache against the float64 oracle: types, head layouts, lengths from nothing to long, masks, values that are not finite."""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B
from decode_parity import DTYPES, cache_values, check_attend, close, f64, normal, random_cache

pytestmark = pytest.mark.gpu

LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 257, 500, 1000, 3]


def run(cache, q, **kw):
    before = cache.weight.clone()
    after = torch.full_like(before, -1.0)
    out, lse = cache.attend(q, weight=after, **kw)
    torch.cuda.synchronize()
    return before, after, out, lse


def check(cache, q, T, lens=None):
    before, after, out, lse = run(cache, q)
    used = torch.zeros_like(before, dtype=torch.bool)
    for s, n in enumerate(cache.lengths.cpu().tolist() if lens is None else lens):
        used[int(cache.layout.offsets[s]):int(cache.layout.offsets[s]) + n] = True
    assert bool((after[~used] == -1.0).all()), "weights of rows that are not in use were written"
    check_attend(cache, q, T, out, lse, before, torch.where(used, after, before), lens)
    return out, lse, after


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (8, 2), (3, 7), (4, 16), (64, 1), (1, 33)])
def test_types_heads_lengths(dtype, d, G, T):
    rng = np.random.default_rng([d, G, T, DTYPES.index(dtype)])
    lens = LENS
    cache = random_cache(rng, dtype, 10, 2, G, d, lens, rooms=[n + (i * 5) % 13 for i, n in enumerate(lens)], before=3)
    check(cache, normal(rng, (10, 2 * G, T, d), dtype), T)


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_segments_are_split(dtype):
    rng = np.random.default_rng(5)
    lens = [20000, 7, 0, 9001]
    cache = random_cache(rng, dtype, 2, 2, 2, 128, lens, rooms=[20011, 500, 40, 15000])
    check(cache, normal(rng, (2, 4, 3, 128), dtype), 3)


@pytest.mark.parametrize("dtype,d,G,T,n", [("bf16", 64, 1, 1, 150001), ("bf16_kv4", 128, 2, 1, 300007), ("f32", 64, 64, 1, 20011), ("f16", 128, 16, 4, 30001), ("bf16_kv8", 64, 3, 10, 40009)])
def test_one_segment_over_the_whole_chip(dtype, d, G, T, n):
    # one segment in as many parts as there are workgroups on the chip, or as the joining launch takes with many queries
    rng = np.random.default_rng(n)
    cache = random_cache(rng, dtype, 1, 1, G, d, [n], rooms=[n + 100])
    check(cache, normal(rng, (1, G, T, d), dtype), T)


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128), ("bf16_kv4", 64)])
@pytest.mark.parametrize("G,T", [(5, 1), (3, 3), (1, 17), (11, 3), (8, 8)])
@pytest.mark.parametrize("n", [130, 700, 2500])
def test_many_queries_on_parts_of_few_rows(dtype, d, G, T, n):
    # threads of the joining launch share the queries; outputs take it several turns
    rng = np.random.default_rng([d, G, T, n])
    cache = random_cache(rng, dtype, 1, 2, G, d, [n, n - 60], rooms=[n + 9, n + 300], before=1)
    check(cache, normal(rng, (1, 2 * G, T, d), dtype), T)


@pytest.mark.parametrize("S", [90, 700])
def test_many_segments_with_long_ones_among_them(S):
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 200, S)
    lens[[3, S // 2, S - 1]] = [9000, 4001, 12000]
    cache = random_cache(rng, "bf16_kv8", S, 1, 4, 64, lens.tolist(), rooms=(lens + 5).tolist())
    check(cache, normal(rng, (S, 4, 2, 64), "bf16_kv8"), 2)


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes(seed):
    rng = np.random.default_rng([77, seed])
    dtype, d = DTYPES[seed % 5], int(rng.choice([64, 128]))
    G = int(rng.choice([1, 2, 3, 4, 5, 8, 12]))
    T = int(rng.integers(1, 64 // G + 1)) if seed % 3 else 1
    B_, Hkv = int(rng.integers(1, 7)), int(rng.choice([1, 2, 3, 8]))
    top = int(2.0 ** rng.uniform(0, 12))
    lens = [int(x) for x in rng.integers(0, top + 1, B_ * Hkv)]
    rooms = [n + int(x) for n, x in zip(lens, rng.integers(0, 400, B_ * Hkv))]
    cache = random_cache(rng, dtype, B_, Hkv, G, d, lens, rooms=rooms, before=int(rng.integers(0, 70)))
    check(cache, normal(rng, (B_, G * Hkv, T, d), dtype), T)


@pytest.mark.parametrize("dtype", DTYPES)
def test_lengths_far_below_the_room(dtype):
    # the parts are planned for the room: they are spread over what is in use
    rng = np.random.default_rng(6)
    lens = [0, 1, 40, 300]
    cache = random_cache(rng, dtype, 2, 2, 4, 64, lens, rooms=[40000, 40000, 40000, 40000])
    check(cache, normal(rng, (2, 8, 2, 64), dtype), 2)


def test_lengths_out_of_range_are_bounded_by_the_room():
    rng = np.random.default_rng(7)
    cache = random_cache(rng, "bf16", 2, 2, 4, 128, [50, 60, 70, 80])
    cache.lengths.copy_(torch.tensor([-5, 1 << 30, 70, -(1 << 31)], dtype=torch.int32))
    check(cache, normal(rng, (2, 8, 1, 128), "bf16"), 1, lens=[0, 60, 70, 0])


def test_no_lengths_is_full_rooms():
    rng = np.random.default_rng(8)
    cache = random_cache(rng, "f16", 1, 3, 2, 128, [33, 64, 1])
    q = normal(rng, (1, 6, 1, 128), "f16")
    out, lse = cache.attend(q, weight=False)
    bare = B.CacheTensors(cache.k, cache.v)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(B.slkv_attend_workspace_bytes(cache.layout, 1, False), dtype=torch.uint8, device="cuda")
    B.slkv_attend_cache(cache.layout, bare, q, o2, ws, l2)
    B.slkv_attend_cache(cache.layout, bare, q, o2, ws, None)          # without lse
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("S", [63, 64, 65, 899, 900, 901, 2000])
def test_segment_tables(S):
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 40, S).tolist()
    lens[S // 2] = 700
    cache = random_cache(rng, "bf16", S, 1, 2, 64, lens, rooms=[n + 9 for n in lens])
    check(cache, normal(rng, (S, 2, 1, 64), "bf16"), 1)


@pytest.mark.parametrize("S", [599, 600, 601, 1199, 1200, 1201])
@pytest.mark.parametrize("split", [False, True])
def test_ends_of_the_large_table(S, split):
    """A launch takes 600 segments: full ones, and a launch of one segment that uses the workspace of the one before, with whole segments in an order of their own and
    with parts in theirs."""
    rng = np.random.default_rng([S, split])
    lens = rng.integers(0, 60, S)
    rooms = lens + 9
    ends = [0, 598, 599, 600, 1198, 1199, 1200]
    for s in ends:
        if s < S:
            lens[s], rooms[s] = (1500 + s, 24000) if split else (40 + s % 7, 90)
    cache = random_cache(rng, "bf16", S, 1, 2, 64, lens.tolist(), rooms=rooms.tolist(), before=4)
    # (without weights the workspace holds the sums of parts, 16 bytes where there are none)
    assert (B.slkv_attend_workspace_bytes(cache.layout, 1, False) > 16) == split
    check(cache, normal(rng, (S, 2, 1, 64), "bf16"), 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [40, 3000])
def test_large_and_concentrated_logits(dtype, n):
    # logits up to some hundreds: references move, most weights vanish
    rng = np.random.default_rng(n)
    cache = random_cache(rng, dtype, 1, 2, 4, 128, [n, n])
    q = normal(rng, (1, 8, 2, 128), dtype)
    check(cache, q * 16, 2)
    check(cache, q * 0, 2)                      # equal weights


def test_fp16_weights_far_below_the_largest():
    # one row takes half of the weight, 30000 rows share the rest, each 2^-16 of the largest or less
    n, d = 30001, 128
    cache = random_cache(np.random.default_rng(1), "f16", 1, 1, 1, d, [n])
    cache.k.zero_()
    cache.k[17] = 1.0
    cache.v.fill_(1.0)
    cache.v[17] = 0.0
    q = torch.full((1, 1, 1, d), float(np.log(30000.0) / np.sqrt(d)), dtype=torch.float16, device="cuda")
    check(cache, q, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16", "bf16_kv8", "bf16_kv4"])
@pytest.mark.parametrize("n", [37, 2000])
def test_values_that_are_not_finite_reach_only_who_sees_them(dtype, n):
    rng = np.random.default_rng(n)
    T = 5
    cache = random_cache(rng, dtype, 1, 4, 2, 64, [n] * 4, rooms=[n + 3] * 4)
    off = cache.layout.offsets

    def put(x, row, value):
        if dtype == "bf16_kv4":
            scale = cache.k_scale if x is cache.k else cache.v_scale
            scale[row, 0] = 255                 # NaN in the first 32 dims
        elif dtype == "bf16_kv8":
            x[row, 5] = 0x7F
        else:
            x[row, 5] = value
    put(cache.v, int(off[0]) + n - 2, float("nan"))     # the last query but one and the last see it
    put(cache.k, int(off[1]) + n - 1, float("nan"))     # the last query sees it
    put(cache.v, int(off[2]) + n - 1, float("inf"))
    put(cache.v, int(off[3]) + n // 2, float("-inf"))   # everybody sees it
    q = normal(rng, (1, 8, T, 64), dtype)
    out, lse, _ = check(cache, q, T)
    assert bool(torch.isfinite(out[0, 0:2, :T - 2]).all()) and bool(torch.isfinite(lse[0, 2:4, :T - 1]).all())


def test_logits_of_minus_infinity():
    # rows of -infinity vanish beside others; a query whose every logit is -infinity has no softmax
    d = 64
    cache = random_cache(np.random.default_rng(2), "f32", 1, 2, 1, d, [50, 40])
    q = torch.ones((1, 2, 1, d), device="cuda")
    cache.k[:25, 0] = float("-inf")
    cache.k[50:, 3] = float("-inf")
    out, lse, w = check(cache, q, 1)
    assert bool(torch.isfinite(out[0, 0]).all()) and bool(torch.isnan(out[0, 1]).all())


def test_queries_that_are_not_finite_stay_alone():
    rng = np.random.default_rng(3)
    cache = random_cache(rng, "bf16", 2, 1, 4, 128, [300, 20])
    q = normal(rng, (2, 4, 2, 128), "bf16")
    q[0, 1, 0, 7] = float("nan")
    out, lse, _ = run(cache, q)[2], run(cache, q)[3], None
    want, wl = cache.attend(torch.nan_to_num(q), weight=False)
    alone = torch.ones((2, 4, 2), dtype=torch.bool, device="cuda")
    alone[0, 1, 0] = False
    close(f64(out)[alone.cpu().numpy()], f64(want)[alone.cpu().numpy()], 2.0 ** -7 * (1 + np.abs(f64(want)[alone.cpu().numpy()])), "others")
    assert bool(torch.isnan(out[0, 1, 0]).all()) and torch.equal(lse[alone], wl[alone])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [3, 40, 5000])
@pytest.mark.parametrize("G,T", [(2, 3), (3, 10), (16, 4)])
def test_queries_without_a_softmax_leave_the_weights_of_rows_behind_them(dtype, n, G, T):
    """A query that holds a NaN makes NaN of the weights of the rows that it sees, and of no others."""
    rng = np.random.default_rng([n, G, T])
    cache = random_cache(rng, dtype, 2, 1, G, 64, [n, n + 1], rooms=[n + 5, n + 40])
    q = normal(rng, (2, G, T, 64), dtype)
    q[0, 0, 0, 3] = float("nan")
    q[1, G - 1, T - 2, 5] = float("nan")
    _, _, w = check(cache, q, T)
    off = cache.layout.offsets
    assert bool(torch.isfinite(w[int(off[0]) + max(n - T + 1, 0):int(off[0]) + n]).all()) and bool(torch.isfinite(w[int(off[1]) + n]))
    assert bool(torch.isnan(w[int(off[1])]))


@pytest.mark.parametrize("n", [20, 5000])
def test_logits_of_minus_infinity_up_to_a_row_that_later_queries_see(n):
    cache = random_cache(np.random.default_rng(4), "f32", 1, 1, 1, 64, [n])
    cache.k[:n - 1, 0] = float("-inf")
    _, lse, w = check(cache, torch.ones((1, 1, 2, 64), device="cuda"), 2)
    assert bool(torch.isnan(lse[0, 0, 0])) and bool(torch.isfinite(lse[0, 0, 1])) and bool(torch.isfinite(w[n - 1])) and bool(torch.isnan(w[0]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_every_time_and_in_place(dtype):
    rng = np.random.default_rng(9)
    cache = random_cache(rng, dtype, 3, 2, 4, 128, [5000, 10, 700, 0, 129, 33], rooms=[6000, 20, 900, 10, 140, 60])
    q = normal(rng, (3, 8, 1, 128), dtype)
    before, after, out, lse = run(cache, q)
    for _ in range(3):
        b2, a2, o2, l2 = run(cache, q)
        assert torch.equal(after, a2) and torch.equal(out, o2) and torch.equal(lse, l2)
    cache.attend(q)                                      # in place
    used = after != -1.0
    assert torch.equal(cache.weight[used], after[used]) and torch.equal(cache.weight[~used], before[~used])
    # without the weights: the same outputs
    o3, l3 = cache.attend(q, weight=False)
    assert torch.equal(out, o3) and torch.equal(lse, l3)
    # weights without a past
    bare = B.CacheTensors(cache.k, cache.v, cache.k_scale, cache.v_scale, cache.lengths)
    ws = torch.empty(B.slkv_attend_workspace_bytes(cache.layout, 1, True), dtype=torch.uint8, device="cuda")
    fresh = torch.zeros_like(after)
    B.slkv_attend_cache(cache.layout, bare, q, o3, ws, l3, fresh)
    want = np.where(used.cpu().numpy(), f64(after) - f64(before), 0)
    close(f64(fresh), want, 2.0 ** -22 * (1 + f64(before)), "fresh weights")


def test_three_streams_at_once():
    """Calls that hold the chip together, a workspace each."""
    rng = np.random.default_rng(14)
    caches = [random_cache(rng, t, 1, 8, 4, 128, [3000 + 100 * i] * 8) for i, t in enumerate(("bf16", "bf16_kv8", "bf16_kv4"))]
    qs = [normal(rng, (1, 32, 1, 128), "bf16") for _ in caches]
    want = [run(c, q)[1:] for c, q in zip(caches, qs)]
    streams = [torch.cuda.Stream() for _ in caches]
    got = [[] for _ in caches]
    for _ in range(20):
        for c, q, s, g in zip(caches, qs, streams, got):
            with torch.cuda.stream(s):
                w = torch.full_like(c.weight, -1.0)
                g.append((w,) + c.attend(q, weight=w))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for one in g for a, b in zip(w, one))


@pytest.mark.parametrize("graph", [False, True])
def test_one_cache_on_three_streams_at_once(graph):
    """Calls that only read the cache, nothing orders them: segments in parts, whose sums pass through a workspace."""
    rng = np.random.default_rng(15)
    cache = random_cache(rng, "bf16", 1, 8, 4, 128, [6000 + 100 * i for i in range(8)])
    qs = [normal(rng, (1, 32, 1, 128), "bf16") for _ in range(3)]
    want = [cache.attend(q, weight=False) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[] for _ in qs]
    torch.cuda.synchronize()
    if graph:
        graphs, outs = [], []
        for q in qs:                                     # captured on one stream, replayed on three
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[0]):
                outs.append(cache.attend(q, weight=False))
            graphs.append(g)
    for _ in range(20):
        for i, (q, s, g) in enumerate(zip(qs, streams, got)):
            with torch.cuda.stream(s):
                if graph:
                    graphs[i].replay()
                    g.append(tuple(x.clone() for x in outs[i]))
                else:
                    g.append(cache.attend(q, weight=False))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for one in g for a, b in zip(w, one))


def test_first_call_inside_a_capture():
    rng = np.random.default_rng(16)
    cache, other = (random_cache(rng, "bf16_kv8", 1, 2, 4, 128, [5000, 40]) for _ in range(2))
    other.attend(normal(rng, (1, 8, 2, 128), "bf16_kv8"))      # (the device has loaded the kernels)
    q, w = normal(rng, (1, 8, 2, 128), "bf16_kv8"), torch.full_like(cache.weight, -1.0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out, lse = cache.attend(q, weight=w)
    for i in range(4):
        q.copy_(normal(rng, q.shape, "bf16_kv8"))
        before, after, o2, l2 = run(cache, q)            # an eager call between the replays
        w.fill_(-1.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(w, after)


def test_scratch_does_not_pile_up():
    rng = np.random.default_rng(17)
    cache = random_cache(rng, "bf16", 1, 8, 4, 64, [20000] * 8)
    torch.cuda.synchronize()
    for T in range(1, 17):
        cache.attend(normal(rng, (1, 32, T, 64), "bf16"))
    held, most = torch.cuda.memory_allocated(), B.slkv_attend_workspace_bytes(cache.layout, 16, True)
    del cache
    # its rows and the largest of 16 workspaces (together they would be 8 times that one); torch may leave up to 1 MiB at the end of each of the five
    assert held - torch.cuda.memory_allocated() < 8 * 20000 * (2 * 128 + 8) + most + (6 << 20)


def test_other_stream():
    rng = np.random.default_rng(10)
    cache = random_cache(rng, "bf16_kv4", 2, 2, 4, 128, [3000, 10, 700, 50])
    q = normal(rng, (2, 8, 1, 128), "bf16_kv4")
    before, after, out, lse = run(cache, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o2, l2, a2 = torch.empty_like(out), torch.empty_like(lse), torch.full_like(after, -1.0)
    cache.attend(q, out=o2, lse=l2, weight=a2, stream=s)
    s.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(after, a2)


def test_rows_beyond_four_gigabytes():
    # fp32 rows of 512 bytes: the second segment's begin above 2^32 bytes
    d, far = 128, (1 << 32) // 512 + 5
    rng = np.random.default_rng(11)
    offsets = np.array([0, far, far + 333], dtype=np.int64)
    k = torch.zeros((far + 333, d), device="cuda")
    v = torch.zeros((far + 333, d), device="cuda")
    k[far:], v[far:] = normal(rng, (333, d), "f32"), normal(rng, (333, d), "f32")
    k[:40], v[:40] = normal(rng, (40, d), "f32"), normal(rng, (40, d), "f32")
    cache = api.Cache("f32", 1, 2, 2, d, offsets, k=k, v=v, lengths=torch.tensor([40, 333], dtype=torch.int32, device="cuda"), weights=False, positions=False)
    q = normal(rng, (1, 2, 1, d), "f32")
    out, lse = cache.attend(q)
    small = api.Cache("f32", 1, 2, 2, d, [0, 40, 373], k=torch.cat((k[:40], k[far:])), v=torch.cat((v[:40], v[far:])), weights=False, positions=False)
    check_attend(small, q, 1, out, lse)


def test_captured_call_follows_the_lengths():
    """Two graphs that share the cache's workspace, replayed in turn while the cache grows, against eager calls."""
    rng = np.random.default_rng(12)
    rooms = [4000, 300, 100, 2000]
    cache = random_cache(rng, "bf16", 2, 2, 4, 128, rooms)
    q1, q2 = normal(rng, (2, 8, 1, 128), "bf16"), normal(rng, (2, 8, 3, 128), "bf16")
    w1, w2 = torch.full_like(cache.weight, -1.0), torch.full_like(cache.weight, -1.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(s):
        for q, w in ((q1, w1), (q2, w2)):
            cache.attend(q, weight=w)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for q, w in ((q1, w1), (q2, w2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(cache.attend(q, weight=w))
        graphs.append(g)
    for lens in ([4000, 300, 100, 2000], [0, 1, 2, 3], [129, 300, 50, 1999], [4000, 0, 100, 640]):
        cache.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        for g, q, w, o in zip(graphs, (q1, q2), (w1, w2), outs):
            w.fill_(-1.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            want_w = torch.full_like(w, -1.0)
            want = cache.attend(q, weight=want_w)
            torch.cuda.synchronize()
            assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1]) and torch.equal(w, want_w)


def test_refusals_of_tensors():
    cache = api.Cache("bf16", 2, 4, 2, 64, [0, 8, 16, 24, 32])
    q = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q[:, :2], q.transpose(1, 2), q[..., :32], q.cpu(), q[0]):
        with pytest.raises(ValueError):
            cache.attend(bad)
    with pytest.raises(ValueError):
        cache.attend(q, out=torch.empty_like(q).float())
    with pytest.raises(ValueError):
        cache.attend(q, weight=torch.empty(31, device="cuda"))
    with pytest.raises(B.SlkvError):
        cache.attend(torch.zeros((2, 4, 33, 64), dtype=torch.bfloat16, device="cuda"))      # 66 queries a segment
