"""slkv_attend_tree against the float64 oracle: types, head layouts, trees, lengths from nothing to long, values that are not finite."""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2508_15806_amd import api
from decode_parity import DTYPES, cache_values, f64, normal, random_cache
from tile_parity import check_outputs

pytestmark = pytest.mark.gpu

LENS = [0, 1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 500, 1000]


def random_parents(rng, B, T):
    return np.array([[-1 if t == 0 or rng.random() < 0.1 else rng.integers(0, t) for t in range(T)] for _ in range(B)])


def truth(bits, T):
    return (bits.cpu().numpy().view(np.uint64)[:, :, None] >> np.arange(T, dtype=np.uint64) & np.uint64(1)).astype(bool)


def check(cache, q, bits, **kw):
    T = q.shape[2]
    out, lse = cache.attend_tree(q, bits, **kw)
    torch.cuda.synchronize()
    k, v = cache_values(cache)
    lens = np.minimum(np.maximum(cache.lengths.cpu().numpy(), 0), np.diff(cache.layout.offsets))
    o, l, terms, spread = decode.attend_tree(f64(q), k, v, cache.layout.offsets, lens, cache.Hkv, truth(bits, T))
    check_outputs(cache.dtype, cache.d, max(1, lens.max()), out, lse, o, l, terms, spread, np.abs(v[np.isfinite(v)]).max(initial=0.0))
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 5), (3, 11), (4, 16), (2, 64), (8, 24)])
def test_types_heads_lengths(dtype, d, G, T):
    rng = np.random.default_rng([d, G, T, DTYPES.index(dtype)])
    cache = random_cache(rng, dtype, 8, 2, G, d, LENS, rooms=[n + (i * 5) % 13 for i, n in enumerate(LENS)], before=3)
    check(cache, normal(rng, (8, 2 * G, T, d), dtype), api.tree_bits(random_parents(rng, 8, T)).cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_any_bits(dtype):
    """Not only trees: tokens that see nothing of the draft, later tokens, bits beyond the draft."""
    rng = np.random.default_rng(3)
    cache = random_cache(rng, dtype, 3, 2, 3, 64, [7, 0, 20, 500, 130, 9], rooms=[9, 4, 20, 510, 140, 40])
    bits = torch.from_numpy(rng.integers(-2 ** 63, 2 ** 63 - 1, (3, 9), dtype=np.int64)).cuda()
    bits[:, 2] = 0
    bits[1, 5] = -1
    out, lse = check(cache, normal(rng, (3, 6, 9, 64), dtype), bits)
    assert bool((out[0, :, 2] == 0).all()) and bool((lse[0, :, 2] == -float("inf")).all())      # 7 and 0 rows, 9 tokens: nothing before the draft


def test_the_chain_is_what_attend_sees():
    rng = np.random.default_rng(4)
    cache = random_cache(rng, "bf16", 2, 2, 2, 128, [300, 50, 8, 1000])
    q = normal(rng, (2, 4, 8, 128), "bf16")
    bits = api.tree_bits(np.tile(np.arange(8) - 1, (2, 1))).cuda()
    out, lse = cache.attend_tree(q, bits)
    want, lse2 = cache.attend(q, weight=False)
    torch.cuda.synchronize()
    np.testing.assert_allclose(f64(lse), f64(lse2), rtol=1e-6, atol=1e-5)
    np.testing.assert_allclose(f64(out), f64(want), rtol=2.0 ** -6, atol=0.02)


@pytest.mark.parametrize("dtype,G,T", [("bf16", 4, 6), ("bf16_kv4", 4, 16), ("f32", 2, 3), ("f16", 4, 32), ("bf16_kv8", 8, 40)])
def test_long_segments_are_split(dtype, G, T):
    rng = np.random.default_rng(5)
    cache = random_cache(rng, dtype, 2, 2, G, 128, [9000, 7, 0, 3001], rooms=[9011, 500, 40, 15000])
    check(cache, normal(rng, (2, 2 * G, T, 128), dtype), api.tree_bits(random_parents(rng, 2, T)).cuda())


@pytest.mark.parametrize("dtype,Hq,T,S,room", [("bf16", 32, 64, 40, 700), ("bf16_kv4", 32, 64, 40, 700), ("bf16_kv8", 64, 64, 80, 300), ("f16", 64, 50, 80, 600), ("bf16_kv4", 16, 16, 128, 900),
                                               ("bf16", 16, 32, 200, 400), ("bf16_kv8", 8, 16, 64, 1500), ("f32", 16, 32, 40, 300)])
def test_enough_queries_for_every_split_of_a_workgroup(dtype, Hq, T, S, room):
    """Sizes at which workgroups of 8 waves are taken, along the queries and along the keys; the first and the last sequence are checked."""
    rng = np.random.default_rng(Hq + T)
    B, d = S // 2, 128
    lens = [room - (i * 7) % 50 for i in range(S)]
    cache = random_cache(rng, dtype, B, 2, Hq // 2, d, lens, rooms=[room] * S)
    q, bits = normal(rng, (B, Hq, T, d), dtype), api.tree_bits(random_parents(rng, B, T)).cuda()
    out, lse = cache.attend_tree(q, bits)
    torch.cuda.synchronize()
    for b in (0, B - 1):
        rows = slice(b * 2 * room, (b + 1) * 2 * room)
        part = api.Cache(dtype, 1, Hq, 2, d, [0, room, 2 * room], k=cache.k[rows], v=cache.v[rows], k_scale=None if cache.k_scale is None else cache.k_scale[rows],
                         v_scale=None if cache.v_scale is None else cache.v_scale[rows], lengths=cache.lengths[2 * b:2 * b + 2])
        k, v = cache_values(part)
        heads = [0, Hq // 2 - 1, Hq // 2, Hq - 1]
        o, l, terms, spread = decode.attend_tree(f64(q[b:b + 1, heads]), k, v, [0, room, 2 * room], lens[2 * b:2 * b + 2], 2, truth(bits[b:b + 1], T))
        check_outputs(dtype, d, room, out[b:b + 1, heads], lse[b:b + 1, heads], o, l, terms, spread, np.abs(v[np.isfinite(v)]).max(initial=0.0))


@pytest.mark.parametrize("S", [90, 700])
def test_many_segments(S):
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 60, S)
    lens[[3, S // 2, S - 1]] = [2000, 1001, 3000]
    cache = random_cache(rng, "bf16_kv4", S, 1, 4, 64, lens.tolist(), rooms=(lens + 5).tolist())
    check(cache, normal(rng, (S, 4, 4, 64), "bf16_kv4"), api.tree_bits(random_parents(rng, S, 4)).cuda())


@pytest.mark.parametrize("seed", range(25))
def test_random_shapes(seed):
    rng = np.random.default_rng([78, seed])
    dtype, Hkv, G, B, T = DTYPES[seed % 5], int(rng.choice([1, 2])), int(rng.choice([1, 2, 3, 5, 8])), int(rng.integers(1, 4)), int(rng.integers(1, 33))
    lens = rng.integers(0, int(rng.choice([30, 200, 2000])), B * Hkv)
    cache = random_cache(rng, dtype, B, Hkv, G, int(rng.choice([64, 128])), lens.tolist(), rooms=(lens + rng.integers(0, 300, B * Hkv)).tolist(), before=int(rng.integers(0, 5)))
    check(cache, normal(rng, (B, Hkv * G, T, cache.d), dtype), api.tree_bits(random_parents(rng, B, T)).cuda())


def test_lengths_outside_the_rooms():
    rng = np.random.default_rng(6)
    cache = random_cache(rng, "bf16", 2, 1, 2, 64, [90, 40], rooms=[90, 60])
    cache.lengths.copy_(torch.tensor([1000, -5], dtype=torch.int32))
    check(cache, normal(rng, (2, 2, 3, 64), "bf16"), api.tree_bits(random_parents(rng, 2, 3)).cuda())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [4, 40])
def test_values_that_are_not_finite(dtype, T):
    """What is in a drafted row reaches the tokens that see it, and no other."""
    rng = np.random.default_rng(T)
    cache = random_cache(rng, dtype, 1, 2, 2, 64, [200, 130], rooms=[210, 150])
    bad = {"f32": float("nan"), "bf16": float("nan"), "f16": float("nan"), "bf16_kv8": 0x7f, "bf16_kv4": 255}[dtype]
    for start, n, x in ((0, 200, 1), (210, 130, 0)):
        row = start + n - T + T // 2 + x
        ((cache.v_scale if x else cache.k_scale) if dtype == "bf16_kv4" else (cache.v if x else cache.k))[row, 0] = bad
    if dtype in ("f32", "bf16", "f16"):
        cache.v[210 + 130 - 1] = float("inf")
    bits = api.tree_bits(random_parents(rng, 1, T)).cuda()
    out, _ = check(cache, normal(rng, (1, 4, T, 64), dtype), bits)
    assert bool(torch.isfinite(out[:, :, :T // 2]).all())


def test_streams_and_graphs():
    """Calls on two streams and in two captured graphs, replayed several times with other work between them, on a cache that grows in between."""
    rng = np.random.default_rng(13)
    cache = random_cache(rng, "bf16", 1, 2, 4, 128, [9000, 3001], rooms=[9040, 9040])
    bits = api.tree_bits(random_parents(rng, 1, 12)).cuda()
    qs = [normal(rng, (1, 8, 12, 128), "bf16") for _ in range(2)]
    cache.attend_tree(qs[0], bits)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cache.attend_tree(q, bits))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        cache.lengths += 1
        want = [[x.clone() for x in cache.attend_tree(q, bits)] for q in qs]
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
            other = cache.attend_tree(qs[i], bits, stream=streams[1 - i])
        torch.cuda.synchronize()
        # (rows that come into use hold NaN: bits are compared)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(other, want[1])), turn
        for i in range(2):
            assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(outs[i], want[i])), turn
