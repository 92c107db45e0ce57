"""slkv_attend_prompt against the float64 oracle: types, head layouts, lengths from nothing to long, histories, strides, values that are not finite."""

import threading

import numpy as np
import pytest
import torch

from oracle import decode
from oracle.prompt import attend_prompt
from paper_2508_15806_amd import api
from decode_parity import HALF_STEP, f64, normal
from tile_parity import check_outputs

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "bf16", "f16", "bf16_kv8"]


def offsets(counts, before=0):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64) + before


def narrow(x, dtype):
    return torch.from_numpy(decode.to_e4m3(f64(x))).cuda() if dtype == "bf16_kv8" else x


def values(x):
    return decode.from_e4m3(x.cpu().numpy()) if x.dtype == torch.uint8 else f64(x)


def inputs(rng, dtype, Hq, Hkv, d, cu_q, cu_k):
    q = normal(rng, (Hq, int(cu_q[-1]), d), dtype)
    k, v = (narrow(normal(rng, (Hkv, int(cu_k[-1]), d), dtype), dtype) for _ in range(2))
    return q, k, v


def check(dtype, Hq, Hkv, d, cu_q, cu_k, q, k, v, out, lse):
    o, l, terms, spread = attend_prompt(f64(q), values(k), values(v), cu_q, cu_k)
    vv = values(v)
    keys = max([1] + np.diff(cu_k).tolist())
    a, b = int(cu_q[0]), int(cu_q[-1])
    check_outputs(dtype, d, keys, out[:, a:b], lse[:, a:b], o[:, a:b], l[:, a:b], terms[:, a:b], spread[:, a:b],
                  np.abs(vv[np.isfinite(vv)]).max(initial=0.0))


def run_and_check(rng, dtype, Hq, Hkv, d, n, m=None, before=0, before_k=0):
    cu_q, cu_k = offsets(n, before), offsets(n if m is None else m, before if m is None else before_k)
    q, k, v = inputs(rng, dtype, Hq, Hkv, d, cu_q, cu_k)
    call = api.PromptCall(dtype, len(n), Hq, Hkv, d, cu_q, None if m is None else cu_k)
    out, lse = call.run(q, k, v)
    torch.cuda.synchronize()
    check(dtype, Hq, Hkv, d, cu_q, cu_k, q, k, v, out, lse)
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (3, 1), (16, 1)])
def test_types_and_heads(dtype, d, Hq, Hkv):
    rng = np.random.default_rng([DTYPES.index(dtype), d, Hq])
    run_and_check(rng, dtype, Hq, Hkv, d, [1, 0, 2, 31, 32, 33, 64, 65, 129, 300], before=5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 16, 17, 40])
def test_few_queries_behind_histories(dtype, n):
    rng = np.random.default_rng([DTYPES.index(dtype), n])
    m = [n, n + 1, 63 + n, 64, 65, 127, 128, 129, 1000 + n, 5000]
    run_and_check(rng, dtype, 8, 2, 128, [min(n, x) for x in m], m, before=2, before_k=7)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16_kv8", 128), ("f32", 64)])
def test_one_sequence(dtype, d):
    rng = np.random.default_rng(d)
    run_and_check(rng, dtype, 4, 2, d, [1500])
    run_and_check(rng, dtype, 2, 1, d, [333], [4000])


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_queries_than_keys(dtype):
    # the first queries see nothing
    rng = np.random.default_rng(9)
    out, lse = run_and_check(rng, dtype, 4, 2, 64, [40, 5, 70, 3], [10, 0, 69, 200])
    assert bool((out[:, :30] == 0).all()) and bool((lse[:, :30] == -float("inf")).all())
    assert bool((out[:, 40:46] == 0).all()) and bool((lse[:, 40:46] == -float("inf")).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng([77, seed])
    Hkv = int(rng.choice([1, 2, 3]))
    G = int(rng.choice([1, 2, 3, 4, 5, 8, 12]))
    B = int(rng.integers(1, 9))
    n = rng.integers(0, int(rng.choice([3, 40, 300])), B)
    m = n + rng.integers(-3, int(rng.choice([1, 90, 1500])), B).clip(-n)
    run_and_check(rng, DTYPES[seed % 4], Hkv * G, Hkv, int(rng.choice([64, 128])), n.tolist(), m.tolist(), int(rng.integers(0, 4)), int(rng.integers(0, 4)))


@pytest.mark.parametrize("dtype,Hq,Hkv,n", [("bf16", 64, 2, [2000]), ("f16", 128, 4, [1000]), ("bf16_kv8", 128, 2, [1000, 3]), ("bf16_kv8", 128, 2, [500]), ("bf16", 64, 2, [1000]), ("f16", 128, 2, [700, 90]),
                                            ("f32", 32, 2, [900])])
def test_enough_queries_for_every_split_of_a_workgroup(dtype, Hq, Hkv, n):
    """Sizes at which workgroups of 8 waves are taken, along the queries and along the keys; some of the heads are checked."""
    rng = np.random.default_rng(Hq + n[0])
    cu = offsets(n)
    q, k, v = inputs(rng, dtype, Hq, Hkv, 128, cu, cu)
    out, lse = api.PromptCall(dtype, len(n), Hq, Hkv, 128, cu).run(q, k, v)
    torch.cuda.synchronize()
    for h in range(Hkv):
        G = Hq // Hkv
        heads = [h * G, h * G + G // 2, h * G + G - 1]
        check(dtype, 3, 1, 128, cu, cu, q[heads], k[h:h + 1], v[h:h + 1], out[heads], lse[heads])


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [("bf16", 64, 8, 128), ("bf16_kv8", 24, 8, 64), ("f16", 40, 8, 128)])
def test_many_tiles_of_unequal_sequences(dtype, Hq, Hkv, d):
    """So many tiles that they are taken in the order of their keys, whatever sequence they are of; sequences without queries, without keys, with fewer keys than queries."""
    rng = np.random.default_rng(Hq)
    n = [300, 0, 650, 17, 411, 128, 40, 5, 1, 222, 333, 700, 260, 0, 90]
    m = [x + y for x, y in zip(n, [0, 30, 0, 400, 90, 0, -10, 0, 0, -222, 1, 64, 0, 0, 1000])]
    cu_q, cu_k = offsets(n, 3), offsets(m, 1)
    q, k, v = inputs(rng, dtype, Hq, Hkv, d, cu_q, cu_k)
    out, lse = api.PromptCall(dtype, len(n), Hq, Hkv, d, cu_q, cu_k).run(q, k, v)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for h in (0, 3, Hkv - 1):
        heads = [h * G, h * G + G - 1]
        check(dtype, 2, 1, d, cu_q, cu_k, q[heads], k[h:h + 1], v[h:h + 1], out[heads], lse[heads])


def test_many_sequences():
    # more than one launch holds
    rng = np.random.default_rng(3)
    n = rng.integers(0, 30, 150)
    n[[10, 80, 149]] = [500, 700, 301]
    run_and_check(rng, "bf16", 4, 2, 64, n.tolist())
    run_and_check(rng, "bf16_kv8", 4, 2, 64, [1] * 150, (n + 1).tolist())


def test_no_tokens():
    for n, m in (([0, 0], None), ([0, 0], [5, 0]), ([3, 0], [0, 0])):
        cu_q, cu_k = offsets(n), offsets(n if m is None else m)
        q, k, v = inputs(np.random.default_rng(1), "bf16", 4, 2, 64, cu_q, cu_k)
        out, lse = api.PromptCall("bf16", 2, 4, 2, 64, cu_q, cu_k).run(q, k, v)
        torch.cuda.synchronize()
        assert out.shape == q.shape and bool((out == 0).all()) and bool((lse == -float("inf")).all())


def test_rows_outside_the_sequences_stay():
    rng = np.random.default_rng(4)
    cu = offsets([30, 20], 10)
    q, k, v = inputs(rng, "bf16", 4, 2, 128, cu, cu)
    out, lse = torch.full_like(q, 7.0), torch.full((4, 60), 7.0, device="cuda")
    api.PromptCall("bf16", 2, 4, 2, 128, cu).run(q, k, v, out, lse)
    torch.cuda.synchronize()
    assert bool((out[:, :10] == 7).all()) and bool((lse[:, :10] == 7).all())
    check("bf16", 4, 2, 128, cu, cu, q, k, v, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8", "f32"])
def test_strides(dtype):
    """Rows inside wider ones, tokens first, heads that share memory."""
    rng = np.random.default_rng(5)
    cu = offsets([70, 1, 130])
    T, Hq, Hkv, d = 201, 6, 2, 64
    q, k, v = inputs(rng, dtype, Hq, Hkv, d, cu, cu)
    want, lse = api.PromptCall(dtype, 3, Hq, Hkv, d, cu).run(q, k, v)
    wide_q = torch.zeros((T, Hq + 3, d + 16), dtype=q.dtype, device="cuda")
    wide_q[:, 1:Hq + 1, 8:d + 8] = q.transpose(0, 1)
    kv = torch.zeros((T, 2, Hkv, d), dtype=k.dtype, device="cuda")
    kv[:, 0], kv[:, 1] = k.transpose(0, 1), v.transpose(0, 1)
    out = torch.full((T, Hq + 1, d + 32), 3.0, dtype=q.dtype, device="cuda")
    got, lse2 = api.PromptCall(dtype, 3, Hq, Hkv, d, cu).run(wide_q[:, 1:Hq + 1, 8:d + 8].transpose(0, 1), kv[:, 0].transpose(0, 1), kv[:, 1].transpose(0, 1),
                                                            out[:, :Hq, 16:d + 16].transpose(0, 1))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    assert bool((out[:, Hq] == 3).all()) and bool((out[:, :, :16] == 3).all()) and bool((out[:, :, d + 16:] == 3).all())
    # one key head for all of them, one query for all tokens
    k1, v1, q1 = k[:1].expand(Hkv, T, d), v[:1].expand(Hkv, T, d), q[:, :1].expand(Hq, T, d)
    out, lse = api.PromptCall(dtype, 3, Hq, Hkv, d, cu).run(q1, k1, v1)
    torch.cuda.synchronize()
    check(dtype, Hq, Hkv, d, cu, cu, q1, k1, v1, out, lse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,m", [(200, 200), (3, 700), (150, 1900)])
def test_values_that_are_not_finite(dtype, n, m):
    """An infinity or NaN in a row reaches the queries that see the row, and no other."""
    rng = np.random.default_rng([n, DTYPES.index(dtype)])
    cu_q, cu_k = offsets([n, n]), offsets([m, m])
    q, k, v = inputs(rng, dtype, 4, 2, 64, cu_q, cu_k)
    bad = float("nan")
    for t, at in ((v, m - 2), (v, m - n // 2), (k, m - 1), (k, m + m - n // 3)):
        t[:, at, 5] = 0x7f if dtype == "bf16_kv8" else bad
    if dtype != "bf16_kv8":
        v[1, m + m - n // 2, 7] = float("inf")
        v[0, m + m - 1] = -float("inf")
    call = api.PromptCall(dtype, 2, 4, 2, 64, cu_q, cu_k)
    out, lse = call.run(q, k, v)
    torch.cuda.synchronize()
    check(dtype, 4, 2, 64, cu_q, cu_k, q, k, v, out, lse)
    assert bool(torch.isfinite(out[:, :max(0, n - n // 2 - 1)]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_logits(dtype):
    """Maxima that move from tile to tile by more than an exponential holds, and logits of thousands."""
    rng = np.random.default_rng(11)
    cu = offsets([600])
    q, k, v = inputs(rng, dtype, 2, 1, 64, cu, cu)
    q *= 30
    k *= torch.linspace(0.01, 30, 600, device="cuda", dtype=k.dtype)[None, :, None]
    out, lse = api.PromptCall(dtype, 1, 2, 1, 64, cu).run(q, k, v)
    torch.cuda.synchronize()
    check(dtype, 2, 1, 64, cu, cu, q, k, v, out, lse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 32768), (1, 1, 3), (1, 1, 100)])
def test_a_long_flat_tail_behind_one_large_key(dtype, d, Hq, Hkv, n):
    """The first key has a logit x of 16.75 or 16.8, all others 0: each of them has less than 2^-24 of the first one's weight, half an ulp of it, all together 2e-3 of it.  Whole prompts whose
    tiles go through all keys, and few queries behind 32765.

    Query i, of the keys 0 .. i: with w = exp(-x), lse = x + ln(1 + i w), out = (v_0 + w sum_j v_j) / (1 + i w).  Products are exact; a logit of 24.2 in base 2 and what the
    log-sum-exp is made of are rounded five times (2^-18 in all); a sum over m keys takes at most one addition for every 32 keys, and 64 more inside steps, between lanes, waves and parts."""
    if dtype == "f32" and n == 32768:
        Hq, Hkv = 4, 4
    m, u, rng = 32768, 2.0 ** -24, np.random.default_rng(d)
    q, k = torch.zeros((Hq, n, d), device="cuda"), torch.zeros((Hkv, m, d), device="cuda")
    of_q, of_k = ((8.0, 8.0), (16.0, 0.75)) if d == 64 else ((16.0, 8.0), (12.0, -0.25))      # products of 134 and 190
    q[:, :, 1], q[:, :, 5] = of_q
    k[:, 0, 1], k[:, 0, 5] = of_k
    x = (of_q[0] * of_k[0] + of_q[1] * of_k[1]) / d ** 0.5
    tdt = api.DTYPES[dtype][1]
    q, k = q.to(tdt), narrow(k.to(tdt), dtype)
    v = narrow(normal(rng, (Hkv, m, d), dtype).abs(), dtype)
    cu_q, cu_k = offsets([n]), offsets([m])
    out, lse = api.PromptCall(dtype, 1, Hq, Hkv, d, cu_q, cu_k).run(q, k, v)
    torch.cuda.synchronize()
    rows = np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, 200)]))
    i = m - n + rows
    w = np.exp(-x)
    assert 0.5 * u < w < u
    sums = (m / 32 + 64) * u
    np.testing.assert_allclose(f64(lse[:, rows]), np.broadcast_to(x + np.log1p(i * w), (Hq, len(rows))), rtol=0, atol=2.0 ** -18 + sums)
    for h in range(Hq):
        vv = values(v[h // (Hq // Hkv)])
        o = (vv[0] + w * (np.cumsum(vv, 0)[i] - vv[0])) / (1 + i * w)[:, None]
        # weights in the queries' type: half a step of each; outputs rounded once; v >= 0, so the sum of p |v| is out itself
        half = HALF_STEP[dtype]
        np.testing.assert_allclose(f64(out[h, rows]), o, rtol=2 * (2.0 ** -18 + sums) + (0 if dtype == "f32" else 2 * half + half ** 2), atol=0)


def test_same_bits_every_time():
    rng = np.random.default_rng(12)
    for n, m in (([700, 40], None), ([2, 9], [6000, 900])):
        cu_q, cu_k = offsets(n), offsets(n if m is None else m)
        q, k, v = inputs(rng, "bf16", 8, 2, 128, cu_q, cu_k)
        call = api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k)
        first = [x.clone() for x in call.run(q, k, v)]
        for _ in range(5):
            again = call.run(q, k, v)
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_streams_and_graphs():
    """Calls of one object on two streams and in two captured graphs, replayed several times with other work between them."""
    rng = np.random.default_rng(13)
    cu_q, cu_k = offsets([4, 30]), offsets([5000, 3001])
    call = api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k)
    sets = [inputs(rng, "bf16", 8, 2, 128, cu_q, cu_k) for _ in range(4)]
    want = [[x.clone() for x in call.run(*s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call.run(*sets[i]))
        graphs.append(g)
    for turn in range(4):
        for o in outs:
            o[0].zero_()
        torch.cuda.synchronize()
        got = []
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
            got.append(call.run(*sets[2 + i], stream=streams[1 - i]))
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])), turn
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[2 + i])), turn


def test_first_call_inside_a_capture():
    """An object whose first call is captured: replays with other work between them, calls outside the graph, and its outputs after the graph is gone."""
    rng = np.random.default_rng(15)
    cu_q, cu_k = offsets([4, 30]), offsets([5000, 3001])
    q, k, v = inputs(rng, "bf16", 8, 2, 128, cu_q, cu_k)
    call, other = (api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k) for _ in range(2))
    want = [x.clone() for x in other.run(q, k, v)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call.run(q, k, v)
    for turn in range(3):
        for x in got:
            x.zero_()
        g.replay()
        again = call.run(q, k, v)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(got, want, again)), turn
    del g, got
    assert all(torch.equal(a, b) for a, b in zip(call.run(q, k, v), want))


def test_two_host_threads_on_one_stream():
    """Calls of one object whose keys are split, from two threads at once, each with inputs and strides of its own."""
    rng = np.random.default_rng(16)
    cu_q, cu_k = offsets([4, 30]), offsets([5000, 3001])
    call = api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k)
    sets = [inputs(rng, "bf16", 8, 2, 128, cu_q, cu_k) for _ in range(2)]
    sets[1] = (sets[1][0].transpose(0, 1).contiguous().transpose(0, 1),) + sets[1][1:]
    want = [[x.clone() for x in api.PromptCall("bf16", 2, 8, 2, 128, cu_q, cu_k).run(*s)] for s in sets]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def several(i):
        try:
            for _ in range(60):
                got[i].append(call.run(*sets[i]))
        except BaseException as e:
            errors.append(e)

    threads = [threading.Thread(target=several, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors and all(torch.equal(a, b) for i in range(2) for x in got[i] for a, b in zip(x, want[i]))
