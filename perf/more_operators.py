"""The attention before and after a prefill's compression, at the sizes it is called at: what is timed when it is timed.

  prompt  a batch of packed prompts (or of the next pieces of them, behind a history) attends to itself, causally: the
          prefill whose keys and values the compression then chooses from
  tree    the queries of a tree of drafted tokens attend to a compacted cache that holds the drafted rows already; which
          drafted rows a token sees are the bits of a 64-bit number
  accept  the drafted tokens that were right stay in the cache, next to each other, the others leave, and the accepted
          tokens' attention weights are added up, for the eviction to rank by

Rows that a call leaves in 8 or 4 bits are read back as 16-bit values (`Cache.rows`).  Capacities differ between heads
as an INF_sc map makes them differ: most heads small, a few large.  Values are synthetic: keys with channels of unequal
size, queries that concentrate on some keys.  Lengths, trees and accepted paths belong to the case, the values to the seed.
"""

import math
import random

import numpy as np
import torch

own = False

QUERY = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "bf16_kv8": torch.bfloat16, "bf16_kv4": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
LOGITS = 1 << 30            # that the plain form holds at a time


def _prompt(name, dtype, B, n, **kw):
    """n: new tokens of a sequence; history: tokens before them; ragged: both differ between sequences; by_token: queries and
    outputs as a projection leaves them, [tokens][heads][d]."""
    c = dict(name=name, op="prompt", dtype=dtype, B=B, Hq=32, Hkv=8, d=128, n=n, history=0, ragged=False, by_token=True, shape=1)
    c.update(kw)
    return c


def _cached(name, op, dtype, B, avg, T, **kw):
    """avg: rows of a head before the draft, on average; T: drafted tokens; A: the longest path that may be accepted."""
    c = dict(name=name, op=op, dtype=dtype, B=B, Hq=32, Hkv=8, d=128, avg=avg, T=T, A=min(T, 6), slack=128, skew=True, shape=1)
    c.update(kw)
    return c


def listed():
    return [
        # a short question, one conversation: latency
        _prompt("prompt_short", "bf16", 1, 130),
        # a batch of packed prompts of 110 to 4000 tokens: the ordinary prefill
        _prompt("prompt_batch", "bf16", 8, 2048, ragged=True),
        # the long prefill that the compression is for
        _prompt("prompt_long", "bf16", 1, 32768),
        # the next piece of a long prompt that is prefilled in pieces: few queries, many keys
        _prompt("prompt_piece", "bf16", 1, 512, history=65024, by_token=False),
        # fp16, short head dimension, three queries a key head, odd lengths
        _prompt("prompt_f16", "f16", 3, 1111, Hq=24, d=64, ragged=True, shape=3),
        # one token of each of 16 conversations whose 8-bit histories nobody has compressed
        _prompt("token_kv8", "bf16_kv8", 16, 1, history=8192, ragged=True, by_token=False, shape=4),
        # fp32, as many key heads as query heads
        _prompt("prompt_f32", "f32", 1, 1024, Hq=4, Hkv=4, d=64, by_token=False),
        # eight drafted tokens of one conversation: latency
        _cached("tree_one_prompt", "tree", "bf16", 1, 128, 8, slack=64),
        # 32 drafted tokens of 16 conversations of 1024 rows a head
        _cached("tree_batch", "tree", "bf16", 16, 1024, 32, shape=2),
        # the 4-bit cache: a large batch, 16 drafted tokens
        _cached("tree_batch_kv4", "tree", "bf16_kv4", 64, 1024, 16, shape=3),
        # up to six of 32 drafted tokens are accepted; up to eight of 64 in an 8-bit cache
        _cached("accept_batch", "accept", "bf16", 16, 1024, 32, shape=4),
        _cached("accept_batch_kv8", "accept", "bf16_kv8", 32, 2048, 64, A=8, shape=5),
    ]


MOST_FLOPS, MOST_BYTES, MOST_LOGITS = 4e12, 240e6, 3e8    # of a drawn case


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["prompt", "prompt", "prompt", "tree", "tree", "accept"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 4, 8])
    c = dict(op=op, Hq=G * Hkv, Hkv=Hkv, d=rng.choice([64, 128, 128]), shape=rng.randrange(1 << 30))
    row = 4 * c["d"]
    if op == "prompt":
        c["dtype"] = rng.choice(["f32", "bf16", "bf16", "bf16", "f16", "bf16_kv8"])
        c["B"] = spread(1, 32)
        c["ragged"], c["by_token"] = rng.random() < 0.7, rng.random() < 0.5
        work_of = 4 * c["d"] * c["Hq"] * c["B"] * (16 if c["dtype"] == "f32" else 1)
        c["n"] = spread(1, max(2, min(40000, math.isqrt(int(MOST_FLOPS / work_of)), int(MOST_BYTES / (2 * row * c["Hq"] * c["B"])))))
        most = min(int(MOST_FLOPS / (work_of * c["n"])), int(MOST_BYTES / (2 * row * Hkv * c["B"])), 130000) - c["n"]
        c["history"] = rng.choice([0, 0, 1]) * spread(1, max(2, most))
        return c
    c["dtype"] = rng.choice(["f32", "bf16", "bf16", "f16", "bf16_kv8", "bf16_kv4", "bf16_kv4"])
    c["B"] = spread(1, 64)
    c["T"] = spread(2, 64)
    c["A"] = rng.randint(1, min(c["T"], 8))
    c["slack"] = spread(8, 300)
    c["skew"] = rng.random() < 0.7
    R = G * c["T"]
    segs = c["B"] * Hkv
    most = min(int(MOST_BYTES / (_row_bytes(c) * segs)), int(MOST_LOGITS / (segs * R)), 80000)
    c["avg"] = spread(8, max(9, most - c["slack"]))
    return c


# ---------------------------------------------------------------- lengths, trees, paths: of the case alone

def _offsets(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int64)


def _lengths(c):
    """(new tokens, keys) of every sequence of a prompt case."""
    r = random.Random(c["shape"])
    new, keys = [], []
    for _ in range(c["B"]):
        n, h = c["n"], c["history"]
        if c["ragged"]:
            n, h = max(1, int(n * r.uniform(0.05, 1.95))), int(h * r.uniform(0.05, 1.95))
        new.append(n)
        keys.append(n + h)
    return new, keys


def _rooms(c):
    """(rows before the draft, room) of every segment."""
    r = random.Random(c["shape"])
    B, Hkv, avg = c["B"], c["Hkv"], c["avg"]
    if c["skew"]:
        fixed = avg // 4
        share = [r.betavariate(0.5, 5) + 1e-3 for _ in range(Hkv)]
        caps = [max(1, fixed + int((avg - fixed) * Hkv * x / sum(share))) for x in share]
    else:
        caps = [avg] * Hkv
    before, rooms = [], []
    for _ in range(B):
        grown = r.randint(8, c["slack"])
        before += [x + grown for x in caps]
        rooms += [x + c["slack"] + c["T"] for x in caps]
    return before, rooms


def _trees(c):
    """What every drafted token sees of the draft, as a number of T bits [B][T], and the accepted paths [B][A], -1 behind their ends.
    Token 0 is the root, a token's parent comes before it; sequences draft up to T tokens (the others see themselves alone).
    An accepted token stands at its place already or behind all places that the path takes, so that a pass can be repeated."""
    r = random.Random(c["shape"] + 1)
    T, A = c["T"], c["A"]
    sees, paths = [], []
    for _ in range(c["B"]):
        m = max(1, min(T, r.randint(T // 2, T)))
        path = [[0]]
        for t in range(1, m):
            up = path[r.randint(max(0, t - 1 - m // 3), t - 1)]
            path.append(up + [t])
        sees.append([sum(1 << t for t in p) for p in path] + [1 << t for t in range(m, T)])
        fit = [p for p in path if len(p) <= A and all(t == i or t >= len(p) for i, t in enumerate(p))]
        best = max(fit, key=len)
        paths.append(best + [-1] * (A - len(best)))
    return sees, paths


def _row_bytes(c):
    """K and V of one row of one head, in the cache."""
    d = c["d"]
    return 2 * {"f32": 4 * d, "bf16": 2 * d, "f16": 2 * d, "bf16_kv8": d, "bf16_kv4": d // 2 + d // BLOCK}[c["dtype"]]


def work(c):
    d, G = c["d"], c["Hq"] // c["Hkv"]
    elt = 4 if c["dtype"] == "f32" else 2
    row = _row_bytes(c)
    if c["op"] == "prompt":
        new, keys = _lengths(c)
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, keys))
        return {"bytes": sum(keys) * c["Hkv"] * row + sum(new) * c["Hq"] * (2 * d * elt + 4), "flops": 4 * d * c["Hq"] * pairs}
    before, _ = _rooms(c)
    S, T = len(before), c["T"]
    if c["op"] == "tree":
        n = sum(before) + S * T
        return {"bytes": n * row + S * G * T * (2 * d * elt + 4) + 8 * c["B"] * T, "flops": 4 * d * G * T * n}
    count = [sum(t >= 0 for t in p) for p in _trees(c)[1]]
    taken = sum(count) * c["Hkv"]
    rows = sum(before) + taken
    pairs = sum(x * count[s // c["Hkv"]] for s, x in enumerate(before))
    back = c["A"] * S * (row + 4 * d) if c["dtype"] in ("bf16_kv8", "bf16_kv4") else 0
    # the accepted rows to their places, the keys, the accepted queries, the weights read and written; what is read back
    return {"bytes": taken * (2 * row + 16) + rows * (row // 2 + 8) + taken * G * (d * elt + 4) + back, "flops": 2 * d * G * pairs}


# ---------------------------------------------------------------- the 4-bit and 8-bit values

def _to_fp4(x):
    """[..., d] values -> (codes uint8 [..., d/2], two values a byte, the first in the low half; exponents uint8 [..., d/32]).
    The exponent of a block is the smallest at which its largest magnitude is at most 7, half a step above the format's 6."""
    b = x.float().reshape(x.shape[:-1] + (x.shape[-1] // BLOCK, BLOCK))
    top = b.abs().amax(-1)
    m, e = torch.frexp(top)                                     # top = m 2^e, m in [0.5, 1): at most 7/8 of 2^e needs 2^(e-3)
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(-127, 127)
    e = torch.where(top > 0, e, torch.full_like(e, -127))
    a = torch.ldexp(b.double(), -e[..., None]).abs()            # exact
    # midpoints go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    code = (code | (torch.signbit(b).to(torch.uint8) << 3)).reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _narrow(c, x):
    """Values -> (the array that holds them, its exponents or None)."""
    if c["dtype"] == "bf16_kv4":
        return _to_fp4(x)
    return (x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if c["dtype"] == "bf16_kv8" else x), None


def _wide(c, x, e=None):
    """The array -> float32 values."""
    if c["dtype"] == "bf16_kv4":
        table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device=x.device)
        v = table[torch.stack((x & 15, x >> 4), -1).reshape(x.shape[:-1] + (-1,)).long()]
        return torch.ldexp(v.reshape(v.shape[:-1] + (-1, BLOCK)), (e.int() - 127)[..., None]).reshape(v.shape)
    return x.view(torch.float8_e4m3fn).float() if c["dtype"] == "bf16_kv8" else x.float()


# ---------------------------------------------------------------- what a program has in hand

def _inputs(c, seed):
    """Tensors of one case, from the seed."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    qt = QUERY[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    channel = torch.exp(0.5 * normal(d))          # keys have a few large channels; queries meet them the other way round
    s = dict(case=c)
    if c["op"] == "prompt":
        new, keys = _lengths(c)
        s["new"], s["keys"], s["cu_q"], s["cu_k"] = new, keys, _offsets(new), _offsets(keys)
        if c["by_token"]:
            s["q"] = (normal(sum(new), Hq, d) * 2 / channel).to(qt).transpose(0, 1)
        else:
            s["q"] = (normal(Hq, sum(new), d) * 2 / channel).to(qt)
        s["k"] = _narrow(c, (normal(Hkv, sum(keys), d) * channel).to(qt))[0]
        s["v"] = _narrow(c, normal(Hkv, sum(keys), d).to(qt))[0]
        return s
    T, A = c["T"], c["A"]
    before, rooms = _rooms(c)
    S, rows = len(before), sum(rooms)
    s["offsets"], s["before"] = _offsets(rooms), before
    s["start"] = torch.from_numpy(s["offsets"][:-1]).to(dev)
    s["at"] = torch.tensor(before, dtype=torch.int32, device=dev)
    s["lengths"] = s["at"] + T
    sees, paths = _trees(c)
    s["sees"] = torch.from_numpy(np.array(sees, dtype=np.uint64).view(np.int64)).to(dev)
    s["path"] = torch.tensor(paths, dtype=torch.int32, device=dev)
    s["pos"] = torch.arange(rows, dtype=torch.int32, device=dev) * 3 + 1
    s["weight"] = torch.rand(rows, generator=g, device=dev).pow_(8) * 50       # few rows have got much of it
    s["k"], s["k_scale"] = _narrow(c, (normal(rows, d) * channel).to(qt))
    s["v"], s["v_scale"] = _narrow(c, normal(rows, d).to(qt))
    s["q"] = (normal(B, Hq, T, d) * 2 / channel).to(qt)
    if c["op"] == "accept":
        s["lse"] = _tree(s)["lse"]                # what the attention on the draft has left
        s["last"] = _offsets([A] * S)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2508_15806_amd import api
        c = s["case"]
        shape = (c["dtype"], c["B"], c["Hq"], c["Hkv"], c["d"])
        if c["op"] == "prompt":
            s["call"] = api.PromptCall(*shape, s["cu_q"], s["cu_k"])
        else:
            s["cache"] = api.Cache(*shape, s["offsets"], k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                   lengths=s["lengths"].clone(), pos=s["pos"], weight=s["weight"])
        if c["op"] == "accept":
            s["sums"] = s["weight"].clone()
    return s


def run(s):
    op = s["case"]["op"]
    if op == "prompt":
        return _own_prompt(s) if own else _attend_prompt(s)
    if op == "tree":
        return _own_tree(s) if own else _tree(s)
    return _own_accept(s) if own else _accept(s)


# ---------------------------------------------------------------- the framework's calls

def _own_prompt(s):
    out, lse = s["call"].run(s["q"], s["k"], s["v"])
    return {"out": out, "lse": lse}


def _own_tree(s):
    out, lse = s["cache"].attend_tree(s["q"], s["sees"])
    return {"out": out, "lse": lse}


def _own_accept(s):
    cache = s["cache"]
    cache.accept(s["path"], s["case"]["T"], at=s["at"], q=s["q"], lse=s["lse"], weight=s["sums"])
    if s["case"]["dtype"] in ("bf16_kv8", "bf16_kv4"):
        k, v, pos = cache.rows(s["last"])
    else:
        k, v, pos = cache.k, cache.v, cache.pos
    return {"k": k, "v": v, "pos": pos, "weight": s["sums"], "lengths": cache.lengths}


# ---------------------------------------------------------------- the plain forms

def _softmax(logit, sees, dim):
    """(weights, log-sum-exp, both 0 and -infinity where nothing is seen) of logits along `dim`; uses up the logits."""
    logit.masked_fill_(~sees, -math.inf)
    top = logit.amax(dim, keepdim=True)
    p = logit.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return p.div_(torch.where(total > 0, total, 1.0)), lse.squeeze(dim)


def _attend_prompt(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=out.device)
    # a sequence at a time, since they differ in length, and no more of its queries than logits fit
    for b, (n, m) in enumerate(zip(s["new"], s["keys"])):
        q0, k0 = int(s["cu_q"][b]), int(s["cu_k"][b])
        k = _wide(c, s["k"][:, k0:k0 + m]).transpose(1, 2).contiguous()
        v = _wide(c, s["v"][:, k0:k0 + m]).contiguous()
        j = torch.arange(m, device=out.device)
        each = max(1, LOGITS // (Hq * m))
        for t in range(0, n, each):
            e = min(n, t + each)
            q = s["q"][:, q0 + t:q0 + e].float().reshape(Hkv, G * (e - t), d)
            logit = torch.bmm(q, k).div_(math.sqrt(d)).reshape(Hkv, G, e - t, m)
            p, l = _softmax(logit, j <= m - n + torch.arange(t, e, device=out.device)[:, None], 3)
            out[:, q0 + t:q0 + e] = torch.bmm(p.reshape(Hkv, G * (e - t), m), v).reshape(Hq, e - t, d).to(out.dtype)
            lse[:, q0 + t:q0 + e] = l.reshape(Hq, e - t)
    return {"out": out, "lse": lse}


def _rows_of(s, most):
    """Row numbers [S, most] of the segments, those beyond the end of the last room as its last."""
    j = torch.arange(most, device=s["start"].device)
    return (s["start"][:, None] + j[None]).clamp(max=int(s["offsets"][-1]) - 1), j


def _values(s, name, at):
    return _wide(s["case"], s[name][at], None if s[name + "_scale"] is None else s[name + "_scale"][at])


def _tree(s):
    c = s["case"]
    B, Hq, Hkv, T, d = c["B"], c["Hq"], c["Hkv"], c["T"], c["d"]
    S, G = B * Hkv, Hq // Hkv
    at, j = _rows_of(s, max(s["before"]) + T)
    q = s["q"].float().reshape(S, G * T, d)
    logit = torch.bmm(_values(s, "k", at), q.transpose(1, 2).contiguous()).div_(math.sqrt(d))         # [S, rows, G T]
    drafted = j[None] - s["at"][:, None]                                                              # [S, rows]
    bits = s["sees"].repeat_interleave(Hkv, 0)[:, None, :] >> drafted.clamp(0, 63)[:, :, None]        # [S, rows, T]
    sees = (drafted < 0)[:, :, None] | (((bits & 1) != 0) & ((drafted >= 0) & (drafted < T))[:, :, None])
    p, lse = _softmax(logit.reshape(S, -1, G, T), sees[:, :, None], 1)
    out = torch.bmm(p.reshape(S, -1, G * T).transpose(1, 2).contiguous(), _values(s, "v", at))
    return {"out": out.reshape(B, Hq, T, d).to(s["q"].dtype), "lse": lse.reshape(B, Hq, T)}


def _accept(s):
    c = s["case"]
    B, Hq, Hkv, T, A, d = c["B"], c["Hq"], c["Hkv"], c["T"], c["A"], c["d"]
    S, G = B * Hkv, Hq // Hkv
    there = torch.cumprod(((s["path"] >= 0) & (s["path"] < T)).int(), 1).bool()                       # [B, A]
    token = torch.where(there, s["path"], 0).long()
    there_s = there.repeat_interleave(Hkv, 0)
    first = (s["start"] + s["at"])[:, None]
    src = (first + token.repeat_interleave(Hkv, 0))[there_s]
    dst = (first + torch.arange(A, device=src.device))[there_s]
    moved = ["k", "v", "pos", "weight"] + (["k_scale", "v_scale"] if s["k_scale"] is not None else [])
    for name in moved:
        s[name][dst] = s[name][src]
    lengths = s["at"] + there_s.sum(1)
    # the accepted tokens' weights, each over the rows up to its own
    at, j = _rows_of(s, max(s["before"]) + A)
    take = token[:, None, :].expand(B, Hq, A)
    q = torch.gather(s["q"], 2, take[..., None].expand(B, Hq, A, d)).float().reshape(S, G * A, d)
    lse = torch.gather(s["lse"], 2, take).reshape(S, 1, G, A)
    logit = torch.bmm(_values(s, "k", at), q.transpose(1, 2).contiguous()).div_(math.sqrt(d)).reshape(S, -1, G, A)
    sees = (j[None, :, None] <= s["at"][:, None, None] + torch.arange(A, device=q.device)) & there_s[:, None]
    p = torch.exp(logit - lse).masked_fill_(~sees[:, :, None], 0.0).sum((2, 3))                       # [S, rows]
    used = j[None] < lengths[:, None]
    weight = s["weight"].clone()
    weight[at[used]] += p[used]
    k, v, pos = s["k"], s["v"], s["pos"]
    if c["dtype"] in ("bf16_kv8", "bf16_kv4"):
        last = ((s["start"] + lengths)[:, None] - A + torch.arange(A, device=q.device)).reshape(-1)
        k, v, pos = _values(s, "k", last).to(s["q"].dtype), _values(s, "v", last).to(s["q"].dtype), s["pos"][last]
    return {"k": k, "v": v, "pos": pos, "weight": weight, "lengths": lengths.int()}


# ---------------------------------------------------------------- from the definition, in 64 bits

def _value64(c, x, e=None):
    """The array -> float64 values."""
    if c["dtype"] == "bf16_kv4":
        codes = torch.stack((x % 16, x // 16), x.dim()).flatten(-2)
        mag = codes & 7                                 # E2M1: 1 exponent-free step of 0.5, then (1 + m/2) 2^(e-1)
        x, m = (mag >> 1).double(), (mag & 1).double()
        v = torch.where(x > 0, (1 + m / 2) * 2.0 ** (x - 1), m / 2)
        return torch.where(codes >= 8, -v, v) * 2.0 ** (e.double().repeat_interleave(BLOCK, -1) - 127)
    return (x.view(torch.float8_e4m3fn) if c["dtype"] == "bf16_kv8" else x).double()


def _exact_prompt(s):
    c = s["case"]
    G, d = c["Hq"] // c["Hkv"], c["d"]
    dev = s["q"].device
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=dev)
    for b in range(c["B"]):
        q0, q1, k0, k1 = (int(x) for x in (s["cu_q"][b], s["cu_q"][b + 1], s["cu_k"][b], s["cu_k"][b + 1]))
        for h in range(c["Hkv"]):
            k, v = _value64(c, s["k"][h, k0:k1]), _value64(c, s["v"][h, k0:k1])
            heads = slice(h * G, h * G + G)
            for i in range(q0, q1, 1024):
                e = min(q1, i + 1024)
                m = k1 - k0 - (q1 - e)                          # keys that the last of these queries sees
                x = torch.matmul(s["q"][heads, i:e].double(), k[:m].t().contiguous()) / d ** 0.5
                far = torch.arange(m, device=dev)[None] - (m - (e - i)) > torch.arange(e - i, device=dev)[:, None]
                x[far.expand_as(x)] = -math.inf
                lse[heads, i:e] = torch.logsumexp(x, 2)
                out[heads, i:e] = torch.matmul(torch.softmax(x, 2), v[:m])
    return {"out": out, "lse": lse}


def _kv64(s, i, n):
    a = int(s["offsets"][i])
    c = s["case"]
    return tuple(_value64(c, s[x][a:a + n], None if s[x + "_scale"] is None else s[x + "_scale"][a:a + n]) for x in ("k", "v"))


def _exact_tree(s):
    c = s["case"]
    B, Hq, Hkv, T, d = c["B"], c["Hq"], c["Hkv"], c["T"], c["d"]
    G = Hq // Hkv
    out = torch.zeros(B, Hq, T, d, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(B, Hq, T, dtype=torch.float64, device=s["q"].device)
    seen = torch.tensor([[[x >> t & 1 for t in range(T)] for x in row] for row in _trees(c)[0]], dtype=torch.bool, device=s["q"].device)
    for i, n in enumerate(s["before"]):
        b, h = divmod(i, Hkv)
        k, v = _kv64(s, i, n + T)
        x = s["q"][b, h * G:(h + 1) * G].double().reshape(G * T, d) @ k.t().contiguous() / d ** 0.5
        x = x.reshape(G, T, n + T)
        x[:, :, n:] = torch.where(seen[b], x[:, :, n:], -math.inf)
        lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, 2)
        out[b, h * G:(h + 1) * G] = torch.softmax(x, 2) @ v
    return {"out": out, "lse": lse}


def _exact_accept(s):
    c = s["case"]
    Hkv, A, d = c["Hkv"], c["A"], c["d"]
    G = c["Hq"] // Hkv
    paths = [[t for t in p if t >= 0] for p in _trees(c)[1]]
    weight = s["weight"].double()
    after = {x: s[x].clone() for x in ("k", "v", "k_scale", "v_scale") if s[x] is not None}
    read = {"k": [], "v": []}
    for i, n in enumerate(s["before"]):
        b, h = divmod(i, Hkv)
        a = int(s["offsets"][i])
        path = paths[b]
        rows = list(range(a, a + n)) + [a + n + t for t in path]     # where the rows that stay come from
        first = a + n
        taken = torch.tensor(rows[n:], device=weight.device)
        for x in after.values():
            x[first:first + len(path)] = x[taken]
        weight[first:first + len(path)] = s["weight"][taken].double()
        m = n + len(path)
        k = _value64(c, after["k"][a:a + m], None if s["k_scale"] is None else after["k_scale"][a:a + m])
        for i_th, t in enumerate(path):
            x = s["q"][b, h * G:(h + 1) * G, t].double() @ k[:n + i_th + 1].t().contiguous() / d ** 0.5
            weight[a:a + n + i_th + 1] += torch.exp(x - s["lse"][b, h * G:(h + 1) * G, t].double()[:, None]).sum(0)
        for x in read:
            e = x + "_scale"
            read[x].append(_value64(c, after[x][a + m - A:a + m], after[e][a + m - A:a + m] if e in after else None))
    if c["dtype"] in ("bf16_kv8", "bf16_kv4"):
        k, v = torch.cat(read["k"]), torch.cat(read["v"])
    else:
        k, v = after["k"].double(), after["v"].double()
    return {"k": k, "v": v, "pos": None, "weight": weight, "lengths": None}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"prompt": _exact_prompt, "tree": _exact_tree, "accept": _exact_accept}[case["op"]](s)
