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


@pytest.mark.parametrize("hd,kv_heads,layers,blocks", [(64, 1, 3, 30000), (128, 3, 1, 5003)])
def test_bounds_of_long_sequences_are_those_of_their_pieces(hd, kv_heads, layers, blocks):
    """Waves that take several blocks in turn: a whole sequence and a part of it that begins and ends inside a block, beside a short one, against calls of at most
    1000 blocks; and an entry of the table that is out of range far behind."""
    g = torch.Generator(device=DEV).manual_seed(blocks)
    kv = torch.zeros(layers, 2, blocks + 5, kv_heads, 16 * hd, dtype=torch.bfloat16, device=DEV)
    kv[:, 0].normal_(generator=g)
    kv[0, 0, 17, 0, 3] = float("inf")
    cache = PagedCache(kv, kv_heads, hd)
    table = torch.full((2, blocks + 5), -1, dtype=torch.int32, device=DEV)
    order = torch.randperm(blocks + 5, generator=g, device=DEV).int()
    table[0, :blocks], table[1, 2:5] = order[:blocks], order[blocks:blocks + 3]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    status = i32(9, 9)
    for first, count in (((0, 32), (16 * blocks, 48)), ((16 * 700 + 5, 33), (16 * (blocks - 900) + 3, 30))):
        cache.bounds.fill_(99)
        cache.store_bounds(table, i32(*first), i32(*count), 16 * blocks, seq_status=status)
        assert status.tolist() == [0, 0]
        got = cache.bounds.clone()
        cache.bounds.fill_(99)
        for s in range(2):
            for at in range(first[s], first[s] + count[s], 16000):
                cache.store_bounds(table[s:s + 1], i32(at), i32(min(16000, first[s] + count[s] - at)), 16000)
        assert torch.equal(got, cache.bounds)
        assert int((got.view(layers, blocks + 5, -1) != 99).any(-1).sum()) == layers * sum((f + c) // 16 - f // 16 for f, c in zip(first, count))
    table[0, blocks - 1] = blocks + 5
    cache.bounds.fill_(99)
    cache.store_bounds(table[:1], i32(0), i32(16 * blocks), 16 * blocks, seq_status=status[:1])
    assert status.tolist() == [2, 0] and bool((cache.bounds == 99).all())
