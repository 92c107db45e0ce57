"""slkv_evict_cache against the oracle's full sort: sets, order, bytes, lengths, ties, weights that are no ordinary numbers."""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B
from decode_parity import DTYPES, random_cache

pytestmark = pytest.mark.gpu


def check(cache, budgets, w, slack=0, positions=True, weights=True, before=0):
    S, Hkv = cache.B * cache.Hkv, cache.Hkv
    off = cache.layout.offsets
    lens = [min(max(n, 0), int(off[s + 1] - off[s])) for s, n in enumerate(cache.lengths.cpu().tolist())]
    most = [min(int(off[s + 1] - off[s]), max(budgets[s % Hkv], w)) for s in range(S)]
    out_off = np.concatenate([[0], np.cumsum([m + slack for m in most])]) + before
    out = api.Cache(cache.dtype, cache.B, cache.Hq, Hkv, cache.d, out_off, positions=positions, weights=weights)
    rows_out = int(out_off[-1])
    for t in (out.k, out.v, out.k_scale, out.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    if out.pos is not None:
        out.pos.fill_(-9)
    if out.weight is not None:
        out.weight.fill_(9.5)
    kept_idx = torch.full((rows_out,), -3, dtype=torch.int32, device="cuda")
    cache.evict(budgets, w, out, kept_idx)
    torch.cuda.synchronize()
    weight = cache.weight.cpu().numpy()
    want = [decode.evict_segment(weight[off[s]:off[s] + lens[s]], w, budgets[s % Hkv]) for s in range(S)]
    assert out.lengths.cpu().tolist() == [len(x) for x in want]
    src = torch.from_numpy(np.concatenate([x + off[s] for s, x in enumerate(want)]).astype(np.int64)).cuda()
    dst = torch.from_numpy(np.concatenate([np.arange(len(x)) + out_off[s] for s, x in enumerate(want)]).astype(np.int64)).cuda()
    assert np.array_equal(kept_idx[dst].cpu().numpy(), np.concatenate(want))
    other = torch.ones(rows_out, dtype=torch.bool, device="cuda")
    other[dst] = False
    assert bool((kept_idx[other] == -3).all())

    def same(a, b, rest):
        if a is None or b is None:
            return
        a, b = (x.view(torch.uint8).reshape(x.shape[0], -1) for x in (a, b))
        assert torch.equal(a[src], b[dst])
        assert bool((b[other] == rest).all()) if rest is not None else True
    same(cache.k, out.k, 0x5A), same(cache.v, out.v, 0x5A)
    same(cache.k_scale, out.k_scale, 0x5A), same(cache.v_scale, out.v_scale, 0x5A)
    same(cache.pos, out.pos, None), same(cache.weight, out.weight, None)
    if out.pos is not None:
        assert bool((out.pos[other] == -9).all())
    if out.weight is not None:
        assert bool((out.weight[other] == 9.5).all())
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("w", [0, 1, 32])
def test_types_lengths_windows(dtype, d, w):
    rng = np.random.default_rng([d, w, DTYPES.index(dtype)])
    lens = [0, 1, 31, 32, 33, 64, 65, 100, 1000, 1023, 1024, 1025, 4096, 4097, 5000, 12]
    cache = random_cache(rng, dtype, 4, 4, 2, d, lens, rooms=[n + 17 for n in lens], before=5)
    check(cache, [0, 31, 64, 700], w, slack=3, before=2)


@pytest.mark.parametrize("n", [8192, 32768, 70001])
@pytest.mark.parametrize("share", [0.01, 0.5, 0.999])
def test_long_histories(n, share):
    rng = np.random.default_rng(n)
    cache = random_cache(rng, "bf16_kv4", 1, 2, 4, 64, [n, n - 5])
    cache.weight.copy_(torch.from_numpy((rng.random(2 * n - 5) ** 12).astype(np.float32)))
    check(cache, [int(n * share), 40], 8)


@pytest.mark.parametrize("n", [50, 3000, 12287 + 5, 12288 + 5, 12289 + 5, 20000])
def test_equal_weights(n):
    rng = np.random.default_rng(n)
    cache = random_cache(rng, "bf16", 1, 4, 1, 64, [n] * 4)
    w = cache.weight.reshape(4, n)
    w[0] = 0.25                                            # all equal
    w[1] = torch.from_numpy(rng.integers(0, 3, n).astype(np.float32))
    w[2] = 0.0
    w[2, ::7] = -0.0                                       # ranks as 0
    w[3] = torch.from_numpy(rng.choice([1.0, np.nextafter(np.float32(1), np.float32(2)), 2.0], n).astype(np.float32))
    check(cache, [n // 3, n // 2, n // 5, n - 7], 5)


@pytest.mark.parametrize("value", [0.0, 1.5, float("nan")])
@pytest.mark.parametrize("n", [40, 100, 700, 1030, 2100, 12300, 40000])
def test_equal_weights_of_a_cache_that_nobody_attended_to(n, value):
    """All ranked weights of every segment are equal, as fill leaves them: no digit is looked for, and waves without ranked rows are at the votes while
    others still read the smallest and largest key."""
    S = 24 if n < 10000 else 8
    rng = np.random.default_rng(n)
    lens = [n - int(x) for x in rng.integers(0, 30, S)]
    cache = random_cache(rng, "bf16", S // 4, 4, 1, 64, lens, rooms=[n] * S)
    rows = cache.rows(np.concatenate([[0], np.cumsum(lens)]))
    cache.fill(rows[0], rows[1], np.concatenate([[0], np.cumsum(lens)]))
    assert all(bool((cache.weight[int(a):int(a) + m] == 0).all()) for a, m in zip(cache.layout.offsets, lens))
    cache.weight.fill_(value)
    for w in (0, 5):
        out = check(cache, [w + 1, 9, n // 2, n - 33], w)
        assert out.lengths.cpu().tolist() == [min(m, max(c, w)) for m, c in zip(lens, [w + 1, 9, n // 2, n - 33] * (S // 4))]


@pytest.mark.parametrize("n", [12289, 36864, 36870, 36871, 50000])
@pytest.mark.parametrize("cap", [7, 300, 9000])
def test_keys_in_lds_and_in_memory(n, cap):
    # w = 6: up to 36864 ranked keys stay in LDS
    rng = np.random.default_rng(n + cap)
    cache = random_cache(rng, "bf16_kv4", 1, 3, 1, 64, [n, 40, n - 1], rooms=[n + 30, 50, n], before=3)
    check(cache, [cap, 20, cap + 1], 6, slack=1)
    cache.weight.copy_((cache.weight * 8).floor())         # many equal weights, some in LDS and some not
    check(cache, [cap, 20, cap + 1], 6)


@pytest.mark.parametrize("around", [0x3F800000, 0x3F800100, 0x3F7FFF00, 0x40000000])
@pytest.mark.parametrize("width,low", [(64, 0.0), (64, -1.0), (300, 1e-30), (2, 0.0), (1000, 0.999)])
def test_many_weights_a_few_steps_apart(around, width, low):
    """Thousands of weights among neighbouring floats on both sides of a digit's end, and one far below that widens the range: the last digit is decided
    among them."""
    n = 9000
    rng = np.random.default_rng([around, width])
    cache = random_cache(rng, "bf16", 1, 4, 1, 64, [n] * 4)
    bits = around + rng.integers(-(width // 2), width - width // 2, 4 * n)
    cache.weight.copy_(torch.from_numpy(bits.astype(np.uint32).view(np.float32)))
    cache.weight[::n] = low
    check(cache, [700, n // 2, n - 300, 5000], 7)


def test_weights_that_are_no_ordinary_numbers():
    n = 2000
    rng = np.random.default_rng(1)
    cache = random_cache(rng, "f16", 1, 3, 1, 64, [n] * 3)
    w = cache.weight.reshape(3, n)
    w[0, ::50] = float("nan")
    w[0, 1::60] = float("inf")
    w[0, 2::70] = -float("nan")
    w[1] = -w[1]
    w[1, ::9] = float("-inf")
    w[2] = w[2] * 1e-42                                    # subnormal
    check(cache, [60, 300, 1000], 0)


def test_lengths_out_of_range():
    rng = np.random.default_rng(2)
    cache = random_cache(rng, "bf16", 1, 4, 1, 64, [100, 100, 100, 100])
    cache.lengths.copy_(torch.tensor([-1, 1 << 30, 60, 100], dtype=torch.int32))
    assert check(cache, [50, 50, 70, 0], 10).lengths.cpu().tolist() == [0, 50, 60, 10]


@pytest.mark.parametrize("S", [64, 65, 239, 240, 241, 900])
def test_segment_tables(S):
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 60, S).tolist()
    cache = random_cache(rng, "bf16_kv4", S, 1, 1, 64, lens, rooms=[n + 4 for n in lens])
    check(cache, [25], 3, slack=1)


@pytest.mark.parametrize("S", [241, 560, 561, 1121])
@pytest.mark.parametrize("longest", [1200, 65535, 65536])
def test_many_segments_around_a_long_one(S, longest):
    rng = np.random.default_rng(S + longest)
    lens = rng.integers(0, 40, S)
    lens[[3, 300 % S, S - 1]] = 700, 1100, 90
    rooms = lens + rng.integers(0, 9, S)
    lens[S // 2], rooms[S // 2] = min(longest, 1300), longest
    cache = random_cache(rng, "bf16_kv4", S, 1, 1, 64, lens.tolist(), rooms=rooms.tolist(), before=11)
    check(cache, [1100], 4, before=7)
    check(cache, [20], 0, slack=2)


def test_without_positions_or_weights():
    rng = np.random.default_rng(3)
    cache = random_cache(rng, "f32", 1, 2, 1, 128, [90, 40])
    check(cache, [30, 30], 2, positions=False, weights=False)


def test_captured_eviction_follows_lengths_and_weights():
    rng = np.random.default_rng(4)
    cache = random_cache(rng, "bf16", 2, 2, 2, 64, [3000, 400, 90, 5])
    budgets, w = [300, 50], 16
    offs = np.concatenate([[0], np.cumsum([300, 50, 90, 16])])
    out, ref = api.Cache("bf16", 2, 4, 2, 64, offs), api.Cache("bf16", 2, 4, 2, 64, offs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cache.evict(budgets, w, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        cache.evict(budgets, w, out)
    for lens in ([3000, 400, 90, 5], [10, 400, 17, 0], [299, 51, 90, 5], [3000, 49, 0, 1]):
        cache.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.weight.copy_(torch.from_numpy(rng.random(cache.rows_in_all, dtype=np.float32)))
        out.k.zero_(), ref.k.zero_(), out.weight.zero_(), ref.weight.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        cache.evict(budgets, w, ref)
        torch.cuda.synchronize()
        assert torch.equal(out.k, ref.k) and torch.equal(out.weight, ref.weight) and torch.equal(out.lengths, ref.lengths)


def test_refusals():
    cache = api.Cache("bf16", 1, 2, 2, 64, [0, 50, 100])
    for offs, status in (([0, 19, 40], 6), ([0, 20, 39], 6)):
        with pytest.raises(B.SlkvError) as e:
            cache.evict([20, 20], 4, api.Cache("bf16", 1, 2, 2, 64, offs))
        assert e.value.status == status
    with pytest.raises(B.SlkvError) as e:
        cache.evict([20, 20], 4, cache)                    # onto itself
    assert e.value.status == 2
    with pytest.raises(B.SlkvError) as e:
        cache.evict([20, 20], 4, api.Cache("f16", 1, 2, 2, 64, [0, 50, 100]))
    assert e.value.status == 2
    with pytest.raises(ValueError):
        cache.evict([20], 4, api.Cache("bf16", 1, 2, 2, 64, [0, 50, 100]))
    with pytest.raises(ValueError):
        cache.evict([20, 20], 4, api.Cache("bf16", 1, 2, 2, 64, [0, 50, 100]), kept_idx=torch.zeros(9, dtype=torch.int32, device="cuda"))
