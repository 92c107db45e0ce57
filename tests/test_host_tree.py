"""CPU-only tests of slkv_attend_tree and slkv_accept_cache: refusals before any GPU call, workspace sizes, the checks of api.Cache, tree_bits, the oracle."""

import contextlib
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B
from test_host_cache import BIG, FAKE, NULL, ODD, arrays, layout


def tree(lay=None, arr=None, T=4, q=FAKE, sees=FAKE, out=FAKE, lse=NULL, ws=FAKE, nbytes=BIG):
    lay, arr = lay or layout(), arrays() if arr is None else arr
    return B.lib().slkv_attend_tree(lay.address, C.addressof(arr), T, q, sees, out, lse, ws, nbytes, None)


def accept(lay=None, arr=None, T=4, A=3, path=FAKE, at=NULL, q=NULL, lse=NULL, w=NULL):
    lay, arr = lay or layout(), arrays() if arr is None else arr
    return B.lib().slkv_accept_cache(lay.address, C.addressof(arr), T, A, path, at, q, lse, w, None)


def test_refused_trees():
    assert tree(T=0) == 2 and tree(T=-3) == 2 and tree(T=65) == 4
    assert tree(lay=layout(d=96)) == 4 and tree(lay=layout(Hq=7)) == 2 and tree(lay=layout(dtype=B.SLKV_BF16_KV_MXFP4)) == 1
    for name in ("q", "sees", "out", "ws"):
        assert tree(**{name: NULL}) == 1 and tree(**{name: ODD}) == 2
    assert tree(lse=ODD) == 2 and tree(arr=arrays(d_k=NULL)) == 1
    lay = layout(offsets=[0, 20000, 20000, 20000, 40000])
    need = B.slkv_tree_workspace_bytes(lay, 4)
    assert need > 4096 and tree(lay=lay, nbytes=need - 1) == 5
    n = C.c_size_t(0)
    assert B.lib().slkv_tree_workspace_bytes(lay.address, 65, C.addressof(n)) == 4 and B.lib().slkv_tree_workspace_bytes(lay.address, 4, None) == 1
    assert B.lib().slkv_tree_workspace_bytes(None, 4, C.addressof(n)) == 1


def test_refused_acceptances():
    assert accept(T=0) == 2 and accept(A=0) == 2 and accept(T=65) == 4 and accept(A=65) == 4
    assert accept(path=NULL) == 1 and accept(path=ODD) == 2 and accept(at=ODD) == 2
    assert accept(arr=arrays(d_lengths=NULL)) == 1
    for some in (dict(q=FAKE), dict(lse=FAKE), dict(w=FAKE), dict(q=FAKE, lse=FAKE), dict(lse=FAKE, w=FAKE), dict(q=FAKE, w=FAKE)):
        assert accept(**some) == 1
    for name in ("q", "lse", "w"):
        assert accept(**dict(dict(q=FAKE, lse=FAKE, w=FAKE), **{name: ODD})) == 2
    assert accept(lay=layout(Hq=1 << 16, Hkv=2)) == 4
    assert accept(lay=layout(d=32)) == 4 and accept(lay=layout(dtype=9)) == 2


def test_rows_of_the_draft_do_not_overlap_the_lengths():
    """d_at may be d_lengths itself, not a part of it: a segment's length would be set while another reads it."""
    lay, lengths = layout(B=4, offsets=[0, 10, 20, 30, 40, 50, 60, 70, 80]), 1 << 20
    for w in (NULL, FAKE):
        for at in (lengths - 16, lengths + 16):
            assert accept(lay=lay, arr=arrays(d_lengths=lengths), at=at, q=w, lse=w, w=w) == 2
            assert b"overlaps" in B.lib().slkv_last_error()


def test_weights_do_not_overlap_those_of_the_cache():
    """d_weight_out may be the cache's weights, not a part of them: a row's weight would be written while another workgroup reads it."""
    lay, weight = layout(offsets=[40, 140, 170, 170, 230]), 1 << 20
    for w in (weight - 189 * 4 // 16 * 16, weight - 16, weight + 16, weight + 189 * 4 // 16 * 16):
        assert accept(lay=lay, arr=arrays(d_weight=weight), q=FAKE, lse=FAKE, w=w) == 2
        assert b"d_weight_out overlaps" in B.lib().slkv_last_error()


def bare_cache(monkeypatch):
    cache = api.Cache.__new__(api.Cache)
    cache.__dict__.update(layout=layout(), B=2, Hq=8, Hkv=2, d=128, query_dtype=torch.bfloat16, device=torch.device("cpu"), weight=torch.zeros(190), rows_in_all=190, _arrays=None,
                          _workspaces={}, _tree_bytes={})
    monkeypatch.setattr(cache, "_on", lambda stream: contextlib.nullcontext(), raising=False)
    return cache


def test_cache_checks_tensors(monkeypatch):
    cache = bare_cache(monkeypatch)
    for name in ("slkv_attend_tree", "slkv_accept_cache"):
        monkeypatch.setattr(B, name, lambda *a, **kw: pytest.fail("the call went through"))
    q, bits, path = torch.zeros((2, 8, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 4), dtype=torch.int64), torch.zeros((2, 3), dtype=torch.int32)
    lse = torch.zeros((2, 8, 4))
    for bad in ((q[:1], bits), (q, bits[:, :3]), (q, bits.int()), (q.half(), bits), (q.transpose(1, 2), bits), (q[0], bits), (q, bits.t().contiguous().t())):
        with pytest.raises(ValueError):
            cache.attend_tree(*bad)
    for args, kw in (((path, 0), {}), ((path, 65), {}), ((path[:1], 4), {}), ((path.long(), 4), {}), ((path[0], 4), {}), ((path, 4), dict(at=path)),
                     ((path, 4), dict(q=q)), ((path, 4), dict(lse=lse)), ((path, 5), dict(q=q, lse=lse)), ((path, 4), dict(q=q, lse=lse.double())),
                     ((path, 4), dict(weight=cache.weight)), ((path, 4), dict(q=q, lse=lse, weight=cache.weight[:5]))):
        with pytest.raises(ValueError):
            cache.accept(*args, **kw)
    cache.weight = None
    with pytest.raises(ValueError, match="weights"):
        cache.accept(path, 4, q=q, lse=lse)


def test_tree_calls_share_scratch_on_one_stream_alone(monkeypatch):
    cache = bare_cache(monkeypatch)
    got = []
    monkeypatch.setattr(B, "slkv_attend_tree", lambda layout_, arrays_, q, sees, out, workspace, lse, stream=None: got.append(workspace))

    def call(stream, capturing=False):
        monkeypatch.setattr(B, "_stream", lambda s: stream)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        cache.attend_tree(torch.zeros((2, 8, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 4), dtype=torch.int64))
        return got[-1]
    apart = [call(0), call(16), call(0, True), call(0, True)]
    spans = sorted((x.data_ptr(), x.data_ptr() + x.nbytes) for x in apart)
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and call(0) is apart[0] and call(16) is apart[1]


def test_tree_bits():
    assert api.tree_bits([-1, 0, 0, 1, 3, -1]).tolist() == [1, 3, 5, 11, 27, 32]
    chain = api.tree_bits(np.arange(64) - 1)
    assert chain[62].item() == 2 ** 63 - 1 and chain[63].item() == -1 and chain.dtype == torch.int64
    assert api.tree_bits([[-1, 0], [-1, -1]]).tolist() == [[1, 3], [1, 2]]
    for bad in ([0], [-1, 1], [-2], [-1, 0.5], list(range(-1, 64))):
        with pytest.raises(ValueError):
            api.tree_bits(bad)


def test_oracle_chain_is_attend():
    """A chain of drafted tokens is what the oracle of attention over a cache computes."""
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((2, 4, 3, 8)), rng.standard_normal((40, 8)), rng.standard_normal((40, 8))
    offsets, lens = [0, 10, 12, 30, 40], [9, 2, 17, 3]
    chain = np.tril(np.ones((3, 3), bool))[None].repeat(2, 0)
    got, want = decode.attend_tree(q, k, v, offsets, lens, 2, chain), decode.attend(q, k, v, offsets, lens, 2, 3)
    for a, b in zip(got[:2], want[:2]):
        np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-14)


def test_oracle_accept():
    assert decode.accept_segment([0, 2, 5, -1, 1], 6, 10, 40) == ([10, 12, 15], 10)
    assert decode.accept_segment([0, 2, 6, 1], 6, 10, 40) == ([10, 12], 10)
    assert decode.accept_segment([0, 2, 5, 1], 6, -2, 40) == ([0, 3], 0)
    assert decode.accept_segment([0, 2, 1], 6, 38, 40) == ([38, 39], 38)
    assert decode.accept_segment([0, 0, 1, 0], 6, 38, 40) == ([38, 38], 38)
