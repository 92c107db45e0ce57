"""CPU-only tests of calls from several host threads."""

import contextlib
import threading
import time

import numpy as np
import pytest
import torch

from paper_2508_15806_amd import api
from paper_2508_15806_amd import binding as B


class Watched(dict):
    """What is stored is looked at as another thread would find it."""

    def __setitem__(self, key, desc):
        assert list(desc.strides) == [256, 64, 64, 640, 64, 640, 256, 64]
        super().__setitem__(key, desc)


def test_a_stored_descriptor_has_its_strides():
    batch = B.PromptBatch(B.SLKV_BF16, 1, 4, 2, 64, [0, 10])
    batch._strided = Watched()
    q, k = torch.zeros((10, 4, 64)).transpose(0, 1), torch.zeros((2, 10, 64))
    batch.with_strides(q, k, k, q)
    assert len(batch._strided) == 1 and list(batch.with_strides(q, k, k, q)[1].strides) == [256, 64, 64, 640, 64, 640, 256, 64]


@pytest.mark.parametrize("op", ["run", "attend", "attend_tree"])
def test_calls_of_one_object_do_not_run_into_each_other(op, monkeypatch):
    """On one stream, in one workspace: a call's launches are all enqueued before another thread's call's."""
    inside, most = [], []

    def library_call(*a, **kw):
        inside.append(1)
        most.append(len(inside))
        time.sleep(0.01)                              # the binding's calls let other threads run
        inside.pop()

    for name in ("slkv_attend_prompt", "slkv_attend_cache", "slkv_attend_tree"):
        monkeypatch.setattr(B, name, library_call)
    monkeypatch.setattr(B, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    on_device = api._OnDevice._set_device
    monkeypatch.setattr(api._OnDevice, "_set_device", lambda self, device: (on_device(self, "cuda:0"), setattr(self, "device", torch.device("cpu"))))
    monkeypatch.setattr(api._OnDevice, "_on", lambda self, stream: contextlib.nullcontext())
    q, k = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((9000, 64), dtype=torch.bfloat16)
    if op == "run":
        x, args = api.PromptCall("bf16", 1, 4, 1, 64, [0, 2], [0, 9000]), (q[0], k[None], k[None])
    else:
        x = api.Cache("bf16", 1, 4, 1, 64, np.array([0, 9000]), k=k, v=k)
        args = (q, torch.zeros((1, 2), dtype=torch.int64)) if op == "attend_tree" else (q,)
    errors = []

    def several():
        try:
            for _ in range(5):
                getattr(x, op)(*args)
        except BaseException as e:
            errors.append(e)

    threads = [threading.Thread(target=several) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and len(most) == 15 and max(most) == 1
