"""CPU-only tests of the calls on a cache: descriptors, refusals before any GPU call, workspace sizes."""

import contextlib
import ctypes as C
import types

import numpy as np
import pytest
import torch

from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B

FAKE, ODD, NULL = 4096, 4100, None
BIG = 1 << 40


def layout(**over):
    p = dict(dtype=B.SLKV_BF16, B=2, Hq=8, Hkv=2, d=128, offsets=[0, 100, 130, 130, 190])
    p.update(over)
    return B.CacheLayout(**p)


def arrays(scaled=False, **over):
    p = dict(d_k=FAKE, d_v=FAKE, d_k_scale=FAKE if scaled else NULL, d_v_scale=FAKE if scaled else NULL, d_lengths=FAKE, d_pos=FAKE, d_weight=FAKE)
    size, reserved = over.pop("struct_size", C.sizeof(B.CacheArrays)), over.pop("reserved", 0)
    p.update(over)
    return B.CacheArrays(size, reserved, *(p[k] for k in ("d_k", "d_v", "d_k_scale", "d_v_scale", "d_lengths", "d_pos", "d_weight")))


def attend(lay=None, arr=None, T=1, q=FAKE, out=FAKE, lse=NULL, weight=NULL, ws=FAKE, nbytes=BIG):
    lay, arr = lay or layout(), arrays() if arr is None else arr
    return B.lib().slkv_attend_cache(lay.address, C.addressof(arr), T, q, out, lse, weight, ws, nbytes, None)


def test_struct_sizes_match_the_header():
    assert C.sizeof(B.CacheDesc) == 6 * 4 + 8 + 8 and C.sizeof(B.CacheArrays) == 8 + 7 * 8


@pytest.mark.parametrize("over,status", [
    (dict(d=96), 4), (dict(Hq=7), 2), (dict(dtype=5), 2), (dict(dtype=-1), 2), (dict(B=0, offsets=[0]), 2),
    (dict(offsets=[0, 100, 90, 130, 190]), 2), (dict(offsets=[-1, 100, 130, 130, 190]), 2), (dict(offsets=[0, 100, 130, 130, 2 ** 31]), 2),
    (dict(Hkv=0, Hq=0, offsets=[0]), 2), (dict(offsets=[0, 0, 2 ** 25 + 1, 2 ** 25 + 1, 2 ** 25 + 1]), 4),
])
def test_descriptors(over, status):
    lay = layout(**over)
    with pytest.raises(B.SlkvError) as e:
        B.slkv_attend_workspace_bytes(lay, 1, True)
    assert e.value.status == status and B.lib().slkv_last_error() != b""


def test_descriptor_struct():
    L, n = B.lib(), C.c_size_t(0)
    lay = layout()
    lay.desc.struct_size = 8
    assert L.slkv_attend_workspace_bytes(lay.address, 1, 0, C.addressof(n)) == 2
    lay = layout()
    lay.desc.reserved[1] = 1
    assert L.slkv_attend_workspace_bytes(lay.address, 1, 0, C.addressof(n)) == 2
    lay = layout()
    lay.desc.h_offsets = None
    assert L.slkv_attend_workspace_bytes(lay.address, 1, 0, C.addressof(n)) == 1
    assert L.slkv_attend_workspace_bytes(None, 1, 0, C.addressof(n)) == 1
    lay = layout()
    assert L.slkv_attend_workspace_bytes(lay.address, 1, 0, None) == 1
    with pytest.raises(ValueError):
        layout(offsets=[0, 1])


def test_layout_keeps_a_copy_of_the_offsets():
    offs = np.array([0, 100, 130, 130, 190], dtype=np.int64)
    lay = layout(offsets=offs)
    before = B.slkv_attend_workspace_bytes(lay, 1, True)
    offs[:] = 5
    assert B.slkv_attend_workspace_bytes(lay, 1, True) == before


def test_attend_refuses_before_touching_the_gpu():
    assert attend(q=NULL) == 1 and attend(out=NULL) == 1 and attend(ws=NULL) == 1
    assert attend(T=0) == 2 and attend(T=17) == 4 and attend(T=1 << 30) == 4          # 4 * 17 queries a segment
    assert attend(lay=layout(Hq=130), T=1) == 4
    for bad in ("q", "out", "lse", "weight", "ws"):
        assert attend(**{bad: ODD}) == 2
    assert attend(nbytes=0) == 5
    need = B.slkv_attend_workspace_bytes(layout(), 1, True)
    assert attend(weight=FAKE, nbytes=need - 1) == 5
    assert B.slkv_attend_workspace_bytes(layout(), 1, False) < need
    for key in ("d_k", "d_v"):
        assert attend(arr=arrays(**{key: NULL})) == 1
        assert attend(arr=arrays(**{key: ODD})) == 2
    assert attend(arr=arrays(d_lengths=ODD)) == 2 and attend(arr=arrays(struct_size=8)) == 2 and attend(arr=arrays(reserved=1)) == 2
    assert attend(arr=arrays(scaled=True)) == 2                                       # scales without MXFP4
    four = layout(dtype=B.SLKV_BF16_KV_MXFP4)
    assert attend(lay=four) == 1 and attend(lay=four, arr=arrays(scaled=True, d_v_scale=NULL)) == 1
    lay = layout()
    assert B.lib().slkv_attend_cache(lay.address, None, 1, FAKE, FAKE, None, None, FAKE, BIG, None) == 1


def test_the_other_calls_refuse_mxfp4():
    lay = B.Layer(B.SLKV_BF16_KV_MXFP4, 1, 8, 2, 128, 16, [0, 100], [40, 40], (128, 12800), (128, 12800))
    with pytest.raises(B.SlkvError) as e:
        B.slkv_compacted_sizes(lay)
    assert e.value.status == 2


def fill(lay=None, arr=None, src=(0, 100, 130, 130, 190), k=FAKE, v=FAKE, pos=FAKE):
    lay, arr = lay or layout(), arrays() if arr is None else arr
    src = None if src is None else np.array(src, dtype=np.int64)
    return B.lib().slkv_fill_cache(lay.address, C.addressof(arr), None if src is None else src.ctypes.data, k, v, pos, None)


def test_fill_refuses_before_touching_the_gpu():
    assert fill(src=None) == 1 and fill(k=NULL) == 1 and fill(v=NULL) == 1 and fill(arr=arrays(d_lengths=NULL)) == 1
    assert fill(src=[0, 101, 131, 131, 191]) == 6                                     # one row too many
    assert fill(src=[0, 10, 5, 30, 60]) == 2 and fill(src=[-1, 10, 15, 30, 60]) == 2
    assert fill(src=[2 ** 31 - 61, 2 ** 31 - 1, 2 ** 31, 2 ** 31, 2 ** 31]) == 2
    assert fill(k=ODD) == 2 and fill(pos=ODD) == 2
    assert fill(arr=arrays(d_pos=NULL)) == 1                                          # positions without a place for them


def append(arr=None, T=1, k=FAKE, v=FAKE, ks=(256, 128, 128), vs=(256, 128, 128), pos=NULL, at=NULL, **over):
    lay = layout(**over)
    arr = arrays() if arr is None else arr
    ks, vs = (None if x is None else (C.c_int64 * 3)(*x) for x in (ks, vs))
    return B.lib().slkv_append_cache(lay.address, C.addressof(arr), T, k, v, None if ks is None else C.addressof(ks), None if vs is None else C.addressof(vs),
                                     pos, at, None)


def test_append_refuses_before_touching_the_gpu():
    assert append(k=NULL) == 1 and append(v=NULL) == 1 and append(ks=None) == 1 and append(arr=arrays(d_lengths=NULL)) == 1
    assert append(T=0) == 2 and append(T=65) == 4
    assert append(ks=(256, 128, 4)) == 2 and append(vs=(-256, 128, 128)) == 2         # 8 bytes; negative
    assert append(k=ODD) == 2 and append(pos=ODD) == 2 and append(at=ODD) == 2
    assert append(pos=FAKE, arr=arrays(d_pos=NULL)) == 1


def test_rows_refuses_before_touching_the_gpu():
    def rows(out=(0, 5, 10, 15, 20), k=FAKE, v=FAKE, pos=NULL, arr=None):
        lay, arr = layout(), arrays() if arr is None else arr
        out = None if out is None else np.array(out, dtype=np.int64)
        return B.lib().slkv_cache_rows(lay.address, C.addressof(arr), None if out is None else out.ctypes.data, k, v, pos, None)
    assert rows(out=None) == 1 and rows(k=NULL) == 1 and rows(v=NULL) == 1 and rows(pos=FAKE, arr=arrays(d_pos=NULL)) == 1
    assert rows(out=[0, 5, 4, 5, 6]) == 2 and rows(k=ODD) == 2


def test_evict_refuses_before_touching_the_gpu():
    far = 1 << 30

    def evict(lay=None, arr=None, out_lay=None, out=None, w=4, budgets=(40, 20), idx=NULL):
        lay = lay or layout()
        out_lay = out_lay or layout(offsets=[0, 40, 60, 100, 120])
        arr = arr or arrays()
        out = out or arrays(**{f: far + i * (1 << 22) for i, f in enumerate(["d_k", "d_v", "d_lengths", "d_pos", "d_weight"])})
        bud = None if budgets is None else np.array(budgets, dtype=np.int32)
        return B.lib().slkv_evict_cache(lay.address, C.addressof(arr), out_lay.address, C.addressof(out), w, None if bud is None else bud.ctypes.data, idx,
                                        None)
    assert evict(w=-1) == 2 and evict(budgets=None) == 1 and evict(budgets=(-1, 3)) == 2
    assert evict(arr=arrays(d_weight=NULL)) == 1
    assert evict(idx=ODD) == 2
    assert evict(out_lay=layout(offsets=[0, 39, 60, 100, 120])) == 6
    assert evict(w=50) == 6                                                            # the latest 50 rows do not fit
    assert evict(out_lay=layout(dtype=B.SLKV_F16, offsets=[0, 40, 60, 100, 120])) == 2
    assert evict(out_lay=layout(Hq=4, offsets=[0, 40, 60, 100, 120])) == 2
    assert evict(out=arrays()) == 2                                                    # the same arrays
    one = dict(d_k=far, d_v=far + (1 << 22), d_lengths=far + (2 << 22), d_pos=far + (3 << 22), d_weight=far + (4 << 22))
    assert evict(out=arrays(**dict(one, d_v=FAKE + 190 * 256 - 16))) == 2              # overlaps by 16 bytes
    assert evict(out=arrays(**dict(one, d_lengths=FAKE))) == 2                         # lengths are read by many workgroups
    assert evict(idx=FAKE) == 2
    assert evict(out=arrays(**dict(one, d_lengths=NULL))) == 1


@pytest.mark.parametrize("budgets,w", [(np.array([2 ** 32 + 40, 20]), 4), (np.array([40, -2 ** 32]), 4), ([40.5, 20], 4), ([40, float("nan")], 4), ([40, 20], 2 ** 32 + 4),
                                       ([40, 20], 2 ** 31)])
def test_evict_refuses_numbers_beyond_32_bits(monkeypatch, budgets, w):
    """A capacity of 2^32 is not one of 0."""
    calls = types.SimpleNamespace(slkv_evict_cache=lambda *a: pytest.fail("the call went through"))
    monkeypatch.setattr(B, "lib", lambda: calls)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    there = types.SimpleNamespace(address=FAKE)
    with pytest.raises(ValueError):
        B.slkv_evict_cache(layout(), there, layout(), there, w, budgets)


def test_evict_takes_whole_numbers_of_any_type(monkeypatch):
    seen = []
    monkeypatch.setattr(B, "lib", lambda: types.SimpleNamespace(slkv_evict_cache=lambda *a: seen.append(((C.c_int32 * 2).from_address(a[5])[:], a[4])) or 0))
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    there = types.SimpleNamespace(address=FAKE)
    for budgets in ([40, 20], (40, 20), np.array([40, 20], dtype=np.int64), np.array([0, 40, 0, 20], dtype=np.int32)[1::2], np.array([40.0, 20.0])):
        B.slkv_evict_cache(layout(), there, layout(), there, np.int64(4), budgets)
    assert seen == [([40, 20], 4)] * 5


def test_a_stream_of_another_device_is_refused():
    cache = api.Cache.__new__(api.Cache)
    cache.device = torch.device("cuda", 0)
    with pytest.raises(ValueError, match="stream"):
        cache._on(types.SimpleNamespace(device=torch.device("cuda", 1)))


def test_calls_of_one_cache_share_scratch_on_one_stream_alone(monkeypatch):
    """Calls that nothing orders have a workspace each: on two streams, and captured ones, whose graphs may be replayed on any."""
    lay = layout()
    cache = api.Cache.__new__(api.Cache)
    cache.__dict__.update(layout=lay, B=2, Hq=8, Hkv=2, d=128, query_dtype=torch.bfloat16, device=torch.device("cpu"), weight=None, rows_in_all=190, _arrays=None,
                          _workspaces={}, _attend_like={})
    monkeypatch.setattr(cache, "_on", lambda stream: contextlib.nullcontext(), raising=False)
    running = []
    monkeypatch.setattr(B, "slkv_attend_cache", lambda layout_, arrays_, q, out, workspace, lse, weight, stream=None: running.append((workspace, out, lse)))

    def attend(stream, T=1, capturing=False):
        monkeypatch.setattr(B, "_stream", lambda s: stream)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        cache.attend(torch.zeros((2, 8, T, 128), dtype=torch.bfloat16), weight=False)
        return running[-1][0]
    apart = [attend(0), attend(0x10), attend(0x20), attend(0, capturing=True), attend(0, capturing=True), attend(0x10, capturing=True)]
    need = B.slkv_attend_workspace_bytes(lay, 1, False)
    for i in range(3):
        spans = sorted((x.data_ptr(), x.data_ptr() + x.nbytes) for one in running for x in (one[i],))
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    assert all(ws.dtype == torch.uint8 and ws.is_contiguous() and ws.nbytes >= need for ws in apart)
    assert attend(0x10) is apart[1] and attend(0) is apart[0]
    # it grows with the largest call
    big = B.slkv_attend_workspace_bytes(lay, 16, False)
    assert attend(0x10, T=16).nbytes >= big and attend(0x10).nbytes >= big and attend(0).nbytes >= need
