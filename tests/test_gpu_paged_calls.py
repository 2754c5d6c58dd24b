"""The operators around the paged cache: tables that go away, calls beside a capture."""
import gc

import pytest
import torch

from paper_2601_17768_amd.paged import PagedCache, Rope

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_rope_is_dropped_while_another_stream_captures():
    g = torch.Generator(device=DEV).manual_seed(1)
    kv = torch.zeros(1, 2, 4, 2, 16 * 64, dtype=torch.bfloat16, device=DEV)
    cache, rope, other = PagedCache(kv, 4, 64), Rope(64, 1e4, 64), Rope(64, 1e4, 64, "interleaved")
    k, q = torch.randn(1, 1, 2, 64, generator=g, device=DEV).bfloat16(), torch.randn(1, 1, 4, 64, generator=g, device=DEV).bfloat16()
    table, lens = torch.arange(4, dtype=torch.int32, device=DEV)[None].contiguous(), torch.tensor([5], dtype=torch.int32, device=DEV)
    step = lambda: cache.append(0, k, k, table, lens, q=q, rope=rope)
    step()
    torch.cuda.synchronize()
    graph, beside = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        out = step()
        with torch.cuda.stream(beside):
            del other
            gc.collect()
    for _ in range(3):
        q.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step())
    rope.close()
    with pytest.raises(ValueError):
        step()
    rope.close()


def test_attention_by_the_largest_scale():
    """Scores of 0 are equal at any scale."""
    g = torch.Generator(device=DEV).manual_seed(2)
    kv = torch.zeros(1, 2, 2, 1, 16 * 64, dtype=torch.bfloat16, device=DEV)
    kv[0, 1] = 3.0
    cache = PagedCache(kv, 2, 64, bounds=False)
    q = torch.randn(1, 1, 2, 64, generator=g, device=DEV).bfloat16()
    table, lens = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), torch.tensor([20], dtype=torch.int32, device=DEV)
    lists = torch.tensor([0, 1], dtype=torch.int32, device=DEV).view(1, 1, 1, 2)
    assert bool((cache.attention(0, q, table, lens, lists, scale=2.0 ** 126) == 3).all())
