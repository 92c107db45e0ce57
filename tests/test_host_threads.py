"""CPU-only tests of calls from several host threads."""

import torch

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
