"""What a binding.Sampling points at lives as long as it does, without a GPU."""
import gc
import weakref

import torch

from paper_2601_17768_amd import binding as B


def test_a_sampling_keeps_its_request_ids(monkeypatch):
    monkeypatch.setattr(B, "_ptr", lambda t, dtype=None: None if t is None else t.data_ptr())
    ids = torch.arange(90)
    at, alive = ids.data_ptr(), weakref.ref(ids)
    sampling = B.make_sampling(1.0, 77, ids)
    assert sampling.request_ids == at
    del ids
    gc.collect()
    assert alive() is not None and alive().tolist() == list(range(90))
    del sampling
    gc.collect()
    assert alive() is None
    assert B.make_sampling(1.0, 77).request_ids is None
