"""Block selection along every way that it picks: rows picked by a wave with its keys in 4, 8 or 16 registers to a lane, by a workgroup from LDS, and through the
workspace by a workgroup that holds 2 or 8 keys to a thread or reads them again; with blocks whose bounds are infinite, fewer and more of them
than a row picks.  Lists are whole numbers: compared for equality.

Sequences share their blocks here (nothing is written), so that many workgroups cost little memory: on 256 CUs scores stay in LDS from 129 workgroups on."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd.paged import PagedCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Shared:
    """Sequences of one context of whole blocks, each with the same physical ones in an order of its own."""

    def __init__(self, seqs, blocks, kv_heads, group, hd, seed=0):
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.seqs, self.blocks, self.kv_heads, self.group, self.hd = seqs, blocks, kv_heads, group, hd
        kv = torch.zeros(1, 2, blocks, kv_heads, 16 * hd, dtype=torch.bfloat16, device=DEV)
        kv[:, 0].normal_(generator=self.g)                        # (in whatever order: random is random)
        self.cache = PagedCache(kv, kv_heads * group, hd)
        ends = torch.tensor([0, blocks - 2, blocks - 1], device=DEV)     # (the first and the last two at the same places in all of them)
        self.table = torch.stack([torch.cat((ends[:1], 1 + torch.randperm(blocks - 3, generator=self.g, device=DEV), ends[1:])) for _ in range(seqs)]).int()

    def infinite(self, ids):
        """Physical blocks whose bounds are to be infinite, for all kv heads."""
        tiles = self.cache.kv[0, 0]
        tiles[ids, :, 5] = torch.tensor([math.nan, math.inf, -math.inf], device=DEV).bfloat16()[torch.arange(len(ids), device=DEV) % 3][:, None]

    def stored(self):
        every = torch.arange(self.blocks, dtype=torch.int32, device=DEV)[None].contiguous()
        zero = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.cache.store_bounds(every, zero, zero + 16 * self.blocks, 16 * self.blocks)
        self.lo, self.hi = (x[0].cpu().double() for x in self.cache.read_bounds(every[0]))

    def check(self, window, budget, sink, recent, rows, most=None):
        """One call; the lists of `rows` of them against the reference, and that no entry keeps what was there."""
        q = torch.randn(self.seqs, window, self.kv_heads * self.group, self.hd, generator=self.g, device=DEV).to(torch.bfloat16)
        len0 = 16 * self.blocks - window
        lens = torch.full((self.seqs,), len0, dtype=torch.int32, device=DEV)
        table = self.table if most is None else torch.nn.functional.pad(self.table, (0, most // 16 - self.blocks), value=-1).contiguous()
        out = torch.full((self.seqs, window, self.kv_heads, budget), -77, dtype=torch.int32, device=DEV)
        self.cache.select(0, q, table, lens, budget, sink, recent, max_context=most, selected=out)
        assert not bool((out == -77).any())
        order = self.table.cpu().long()
        every = [(s, i, h) for s in range(self.seqs) for i in range(window) for h in range(self.kv_heads)]
        for s, i, h in every[::max(1, len(every) // rows)]:
            lo, hi = self.lo[order[s], h], self.hi[order[s], h]
            want = ref.select(q[s, i, h * self.group:(h + 1) * self.group].cpu(), lo, hi, (len0 + i) // 16, budget, sink, recent)
            assert out[s, i, h].tolist() == want, (s, i, h)


# (sequences, blocks, kv heads, group, hd, longest context of the call or None for its own): keys to a lane of a wave 4, 8, 16; a workgroup from LDS;
# through the workspace 2 and 8 keys to a thread, and any number of them
WAYS = {"wave_4": (3, 200, 2, 2, 64, None), "wave_8": (3, 400, 2, 3, 128, None), "wave_16": (33, 900, 4, 2, 64, None), "workgroup": (33, 1300, 4, 1, 128, None),
        "workspace_2": (2, 1300, 2, 4, 64, None), "workspace_8": (2, 1300, 2, 4, 64, 3000 * 16), "workspace_any": (2, 1300, 2, 4, 128, 9000 * 16)}


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("k,more", [(1, 1), (4, -1), (4, 0), (4, 1), (4, None), (61, 0), (61, 1), (61, 40), (61, None)])
def test_select_where_blocks_have_infinite_bounds(way, k, more):
    """k blocks to pick, k + more of them infinite (None: every one): those come first, the lowest of them where they are too many."""
    seqs, blocks, kv_heads, group, hd, most = WAYS[way]
    w = Shared(seqs, blocks, kv_heads, group, hd, seed=k)
    w.infinite(1 + torch.randperm(blocks - 3, generator=w.g, device=DEV)[:blocks if more is None else k + more])
    w.stored()
    w.check(1, k + 3, 1, 2, 12, most)


def test_equal_keys_in_every_way():
    """All blocks alike, so that every round of the pick finds nothing to tell apart: the lowest ones."""
    for seqs, blocks, kv_heads, group, hd, most in WAYS.values():
        w = Shared(seqs, blocks, kv_heads, group, hd)
        w.cache.kv[0, 0] = w.cache.kv[0, 0, :1].clone()
        w.stored()
        w.check(1, 9, 2, 3, 8, most)


def test_scores_of_more_than_the_workspace_holds_go_through_it_in_turn():
    """20 windows of 64 rows over 131072 positions, 8 kv heads: 16 of them fit at once.  Every sequence gets what it gets alone, status and rows that take no part among it."""
    w = Shared(20, 8192, 8, 1, 64)
    w.stored()
    assert B.llm42_kv_select_workspace_bytes(w.cache.heads, 20, 64, 131072, 7) == 256 << 20
    w.check(64, 7, 1, 2, 14)
    q = torch.randn(20, 64, 8, 64, generator=w.g, device=DEV).to(torch.bfloat16)
    lens = torch.randint(0, 131000, (20,), generator=w.g, device=DEV, dtype=torch.int32)
    valid = torch.randint(0, 65, (20,), generator=w.g, device=DEV, dtype=torch.int32)
    lens[[3, 18]] = torch.tensor([-1, 131009], dtype=torch.int32, device=DEV)
    valid[18] = 64
    table = w.table.clone()
    table[17, 0], lens[17], valid[17] = -1, 500, 3
    status = torch.full((20,), 9, dtype=torch.int32, device=DEV)
    out = torch.full((20, 64, 8, 7), -77, dtype=torch.int32, device=DEV)
    w.cache.select(0, q, table, lens, 7, n_valid=valid, selected=out, seq_status=status)
    alone, one = torch.full_like(out, -77), torch.full_like(status, 9)
    for s in range(20):
        w.cache.select(0, q[s:s + 1], table[s:s + 1], lens[s:s + 1], 7, n_valid=valid[s:s + 1], selected=alone[s:s + 1], seq_status=one[s:s + 1])
    assert torch.equal(out, alone) and torch.equal(status, one)
    assert status.tolist() == [1 if s in (3, 18) else 2 if s == 17 else 0 for s in range(20)]
    assert bool((out[[3, 17, 18]] == -77).all())


@pytest.mark.parametrize("hd,kv_heads,group,window,blocks", [(128, 4, 3, 1, 12288), (64, 4, 1, 1, 12279), (128, 4, 4, 4, 3072), (64, 3, 1, 17, 768), (128, 2, 2, 9, 1536)])
def test_the_most_scores_that_lds_holds(hd, kv_heads, group, window, blocks):
    """48 KiB of them, for one row or up to 16, beside the records that are turned there; rows picked by waves and by the workgroup, one after the other."""
    seqs = 129 // kv_heads + 1
    w = Shared(seqs, blocks, kv_heads, group, hd, seed=window)
    w.infinite(torch.randperm(blocks, generator=w.g, device=DEV)[:5])
    w.stored()
    assert B.llm42_kv_select_workspace_bytes(w.cache.heads, seqs, window, 16 * blocks, 50) == 0
    w.check(window, 50, 1, 2, 24)
    w.check(window, 3, 0, 1, 12)
