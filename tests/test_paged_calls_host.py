"""Calls around the paged cache that are refused, or do nothing, without a GPU."""
import ctypes
import gc

import pytest
import torch

from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd.paged import PagedCache, Rope


def test_model_heads_refuses():
    lib, heads = B.load_library(), B.Heads()
    assert lib.llm42_model_heads(None, ctypes.byref(heads)) == B.LLM42_EINVAL


def test_the_sparse_step_compares_heads_by_their_numbers(monkeypatch):
    """One kv head of 128 features and two of 64 take the same bytes of cache, but not of bounds."""
    model, given, done = B.Heads(2, 4, 2, 64), B.Heads(2, 4, 1, 128), []
    blocks, table = 4, torch.zeros((1, 4), dtype=torch.int32)
    kv = torch.zeros(B.llm42_heads_kv_bytes(model, blocks), dtype=torch.uint8)
    assert B.llm42_heads_kv_bytes(given, blocks) == kv.numel() and B.llm42_kv_bounds_bytes(given, blocks) < B.llm42_kv_bounds_bytes(model, blocks)
    monkeypatch.setattr(B, "_all_here", lambda *a: None)
    monkeypatch.setattr(B, "_kv_view", lambda m, base, n, bt, s: B.KVCache(None, n, None, bt.shape[1]))
    monkeypatch.setattr(B, "llm42_kv_bytes", lambda m, n: kv.numel())
    monkeypatch.setattr(B, "llm42_model_heads", lambda m: model, raising=False)
    monkeypatch.setattr(B, "load_library", lambda: pytest.fail("the step was called") if done else B._lib)
    bounds, one = torch.zeros(B.llm42_kv_bounds_bytes(given, blocks), dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)
    done.append(1)
    monkeypatch.setattr(B, "_asked", lambda call, *a: kv.numel())
    with pytest.raises(ValueError, match="not the model's"):
        B.llm42_decode_step_sparse(1, given, kv, blocks, table, bounds, 2, 0, 1, one, one, 16, one, torch.zeros(256, dtype=torch.uint8))


@pytest.mark.parametrize("seqs,most", [(2 ** 25, 1), (2 ** 24, 17), (1, 16 * (2 ** 25 - 1) - 14)])
def test_bounds_store_refuses_what_is_more_threads_than_a_launch_takes(seqs, most):
    """2 kv heads: 2^26 waves, in workgroups of four, are 2^32 threads."""
    heads, kv = B.Heads(2, 8, 2, 128), B.KVCache(4096, 4, 4096, 4)
    assert seqs * ((most + 14) // 16 + 1) * 2 == 2 ** 26
    assert B.load_library().llm42_kv_bounds_store(ctypes.byref(heads), -1, ctypes.byref(kv), 4096, 4096, 4096, seqs, most, None, None) == B.LLM42_EINVAL


@pytest.mark.parametrize("seqs,most,kv_heads", [(2 ** 30, 2 ** 31 - 30, 1024), (2 ** 31 - 1, 2 ** 31 - 1, 1024), (2 ** 31 - 1, 1, 1), (1, 2 ** 31 - 1, 1)])
def test_bounds_store_refuses_sizes_whose_product_passes_64_bits(seqs, most, kv_heads):
    heads, kv = B.Heads(2, kv_heads, kv_heads, 64), B.KVCache(4096, 4, 4096, 4)
    assert B.load_library().llm42_kv_bounds_store(ctypes.byref(heads), -1, ctypes.byref(kv), 4096, 4096, 4096, seqs, most, None, None) == B.LLM42_EINVAL


def unmade_rope(handle):
    rope = Rope.__new__(Rope)
    rope.rot_dim, rope.max_position, rope.handle, rope.device = 64, 128, handle, 0
    return rope


def test_append_refuses_a_closed_rope(monkeypatch):
    """(The library takes a null handle for "no rotation".)"""
    cache, called = PagedCache(torch.zeros(1, 2, 2, 1, 16 * 64, dtype=torch.bfloat16), 1, 64, bounds=False), []
    monkeypatch.setattr(B, "llm42_kv_append", lambda *a: called.append(a))
    k, lens, table = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="closed"):
        cache.append(0, k, k, table, lens, rope=unmade_rope(None))
    assert not called
    cache.append(0, k, k, table, lens)
    assert len(called) == 1


def test_a_dropped_rope_neither_waits_nor_frees(monkeypatch):
    """A finalizer runs whenever its object is collected, while another stream captures as well; the table is given back with the next one that is closed, on its own
    device."""
    calls = []
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: calls.append(("wait", device)))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(B, "llm42_rope_destroy", lambda handle: calls.append(("free", handle)))
    first, second = unmade_rope(11), unmade_rope(12)
    first.device = 3
    del first
    gc.collect()
    assert not calls
    second.close()
    assert sorted(calls[i:i + 2] for i in (0, 2)) == [[("wait", 0), ("free", 12)], [("wait", 3), ("free", 11)]]
    second.close()
    del second
    gc.collect()
    assert len(calls) == 4
    captured = unmade_rope(13)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="capture"):
        captured.close()
    assert len(calls) == 4 and captured.handle == 13
    captured.handle = None


def test_the_selections_workspace_has_a_ceiling():
    """256 MiB, or what a sequence alone takes; it grows with the context, and never falls."""
    need = lambda heads, *a: B.llm42_kv_select_workspace_bytes(heads, *a)
    small, large = B.Heads(1, 32, 8, 128), B.Heads(1, 1024, 1024, 64)
    assert need(small, 8, 512, 131072, 64) == need(small, 32768, 2, 131072, 64) == 256 << 20
    assert need(small, 2, 1, 131072, 64) == 2 * 4 * 8 * 8192
    assert need(large, 1, 512, 2 ** 20, 64) == need(large, 128, 512, 2 ** 20, 64) == 4 * 512 * 1024 * 2 ** 16
    for seqs, window in ((1, 1), (3, 64), (128, 1), (128, 512)):
        sizes = [need(small, seqs, window, 1000 * 2 ** i + j, 64) for i in range(20) for j in (0, 1, 300)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("scale", [2.0 ** 126 * 1.01, 3.4e38])
def test_sparse_attention_refuses_a_scale_that_overflows_in_base_2(scale):
    heads, kv = B.Heads(2, 8, 2, 128), B.KVCache(4096, 4, 4096, 4)
    assert B.load_library().llm42_kv_sparse_attention(ctypes.byref(heads), 0, ctypes.byref(kv), 4096, 1024, 4096, 2, None, 3, 64, 4096, 8, scale, 8192, 1024,
                                                      None, None, 0, None) == B.LLM42_EINVAL
