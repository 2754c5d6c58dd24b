"""The operators around the paged bf16 cache on the GPU against their definitions in float64: appending to the last position, bounds and selections exactly,
attention over lists of every kind, and all of them together.

Tolerances.  A bf16 result is off by half a step, 2^-8 of it, and by the fp32 arithmetic before.  append: the norm's sum of up to 128 squares, its root,
quotient and products are each off by 2^-24 of themselves, in all less than 2^-19 of a value (no sum has more than 20 dependent steps); a rotation adds products
with cos and sin that are off by 2^-24 of the larger of the pair: 2^-18 of the row's largest magnitude covers both.  attention: a score is a sum of up to
128 exact products, off by less than 2^-20 of the sum of their magnitudes, which is below 64 here (scaled): a weight is off by less than 2^-13 of itself, with its two bf16
parts (2^-17) included; so is the sum of weights: 2^-12 of the weighted magnitudes of V covers the output."""
import math

import numpy as np
import pytest
import torch

import paged_reference as ref
from helpers import wl
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd import kv_layout
from paper_2601_17768_amd.paged import PagedCache, Rope

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)
LLAMA3 = dict(kind="llama3", factor=8.0, low_freq_factor=1.0, high_freq_factor=4.0, original_max_position=64)
YARN = dict(kind="yarn", factor=4.0, beta_fast=32.0, beta_slow=1.0, original_max_position=256)


class World:
    """Sequences of some lengths in a paged cache whose blocks lie in no order, with room for `more` positions behind each."""

    def __init__(self, lens, kv_heads=2, group=2, hd=64, layers=2, more=0, seed=0, bounds=True, mirror_v=False):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.g, self.group, self.hd, self.kv_heads = [int(n) for n in lens], g, group, hd, kv_heads
        table, blocks = wl.make_block_table(wl.rng_for(seed, 5), [max(n + more, 1) for n in self.lens], 16, spare_blocks=3)
        self.table, self.bt = table, torch.as_tensor(table, device=DEV)
        kv = torch.randn(layers, 2, blocks, kv_heads, 16 * hd, generator=g).to(torch.bfloat16)
        self.k, self.v = [], []
        for s, n in enumerate(self.lens):
            k = torch.randn(layers, n, kv_heads, hd, generator=g) * torch.exp2(torch.randint(-2, 3, (kv_heads, hd), generator=g).float())
            v = torch.randn(layers, n, kv_heads, hd, generator=g)
            self.k.append(k.to(torch.bfloat16))
            self.v.append(v.to(torch.bfloat16))
            if n:
                kv_layout.write_tokens(kv, torch.as_tensor(table[s]), self.k[s], self.v[s])
        self.cache = PagedCache(kv.to(DEV), kv_heads * group, hd, bounds=bounds)

    def queries(self, window):
        return torch.randn(len(self.lens), window, self.kv_heads * self.group, self.hd, generator=self.g).to(torch.bfloat16)

    def bounds(self, layer, s):
        """[blocks][kv head][feature] of the whole blocks, float64."""
        lo, hi = [], []
        for b in range(self.lens[s] // 16):
            pairs = [ref.bounds(self.k[s][layer, 16 * b:16 * b + 16, h]) for h in range(self.kv_heads)]
            lo.append(torch.stack([x for x, _ in pairs]))
            hi.append(torch.stack([y for _, y in pairs]))
        empty = torch.zeros(0, self.kv_heads, self.hd, dtype=torch.float64)
        return (torch.stack(lo), torch.stack(hi)) if lo else (empty, empty)


def rows_in(values, extra, dtype):
    """The rows [seqs, window, heads, hd] inside a wider matrix: `extra` features before and behind them, on the device."""
    n, w, h, d = values.shape
    wide = torch.full((n, w, h * d + 2 * extra), 7.0, dtype=dtype, device=DEV)
    wide[:, :, extra:extra + h * d] = values.reshape(n, w, h * d).to(dtype).to(DEV)
    return wide[:, :, extra:extra + h * d].unflatten(-1, (h, d)), wide


APPENDS = {
    "one_token": dict(lens=[37], window=1),
    "ragged_inter_part": dict(lens=[0, 5, 16, 31, 100], window=13, valid=[13, 0, 1, 7, 12], rope=(32, 1e4, "interleaved", dict(kind="linear", factor=4.0)),
                              norms=True, dtype=torch.float32),
    "odd_pairs_of_128": dict(lens=[3, 250], window=33, hd=128, group=3, kv_heads=3, rope=(54, 5e5, "half", LLAMA3), norms=True),
    "whole_128": dict(lens=[1, 15, 16, 17, 127], window=16, hd=128, group=4, rope=(128, 5e5, "half", LLAMA3)),
    "yarn_factor_given": dict(lens=[490], window=40, hd=128, group=16, kv_heads=1, rope=(64, 1e6, "half", dict(YARN, attention_factor=1.25)), norms=True,
                              dtype=torch.float32),
    "yarn": dict(lens=[200, 11], window=5, rope=(64, 1e4, "interleaved", YARN)),
    "two_features": dict(lens=[20], window=3, rope=(2, 1e4, "half", dict(kind="none")), group=5, kv_heads=1),
    "no_rope": dict(lens=[9, 40], window=20, rope=None, norms=True),
    "neither_no_q": dict(lens=[9, 40], window=20, rope=None, q=False),
    "long_window": dict(lens=[0, 7], window=512, rope=(64, 1e4, "half", dict(kind="none")), norms=True, kv_heads=1),
    "in_place": dict(lens=[30, 2], window=4, rope=(64, 1e4, "half", dict(kind="none")), norms=True, in_place=True),
    "wide_rows": dict(lens=[30, 2], window=4, rope=(64, 1e4, "half", dict(kind="none")), extra=8, hd=128),
}


@pytest.mark.parametrize("name", APPENDS)
def test_append(name):
    c = dict(window=1, kv_heads=2, group=2, hd=64, rope=(64, 1e4, "half", dict(kind="none")), norms=False, dtype=torch.bfloat16, q=True, valid=None,
             in_place=False, extra=0)
    c.update(APPENDS[name])
    w = World(c["lens"], c["kv_heads"], c["group"], c["hd"], more=c["window"])
    n, window, heads, layer = len(c["lens"]), c["window"], c["kv_heads"] * c["group"], 1
    make = lambda h: (torch.randn(n, window, h, c["hd"], generator=w.g) * (0.5 + torch.rand(h, c["hd"], generator=w.g))).to(c["dtype"])
    q, k, v = make(heads), make(c["kv_heads"]), make(c["kv_heads"])
    gains = [(1 + 0.2 * torch.randn(c["hd"], generator=w.g)).to(torch.bfloat16) if c["norms"] else None for _ in range(2)]
    valid = c["valid"] or [window] * n
    rope = None
    if c["rope"]:
        rot, theta, layout, scaling = c["rope"]
        rope = Rope(rot, theta, 600, layout, scaling)
    before, status = w.cache.kv.clone(), i32([-1] * n)
    dq, _ = rows_in(q, c["extra"], c["dtype"])
    out, out_wide = (dq, None) if c["in_place"] else rows_in(torch.full(q.shape, 9.0), c["extra"], torch.bfloat16)
    on = lambda t: None if t is None else t.to(DEV)
    w.cache.append(layer, rows_in(k, c["extra"], c["dtype"])[0], rows_in(v, 2 * c["extra"], c["dtype"])[0], w.bt, i32(c["lens"]),
                   q=dq if c["q"] else None, q_out=out if c["q"] else None, n_valid=i32(valid) if c["valid"] else None, rope=rope, q_norm=on(gains[0]),
                   k_norm=on(gains[1]), eps=1e-5, seq_status=status)
    assert status.tolist() == [0] * n
    want, tol = before.cpu().double(), torch.zeros(before.shape, dtype=torch.float64)
    for s in range(n):
        for i in range(window):
            pos = c["lens"][s] + i
            if i >= valid[s]:
                if c["q"] and not c["in_place"]:
                    assert bool((out[s, i] == 9).all())
                if c["in_place"]:
                    assert torch.equal(out[s, i].cpu(), q[s, i])
                continue
            if c["q"]:
                r = ref.turned(q[s, i], pos, gains[0], 1e-5, c["rope"])
                lim = r.abs() * 2.0 ** -8 + 2.0 ** -18 * r.abs().amax(-1, keepdim=True)
                assert bool(((out[s, i].cpu().double() - r).abs() <= lim).all()), (s, i)
            kr = ref.turned(k[s, i], pos, gains[1], 1e-5, c["rope"])
            one = lambda t: t[None, None].expand(2, 1, *t.shape)
            for dst, a, b in ((want, kr, v[s, i].to(torch.bfloat16).double()),
                              (tol, kr.abs() * 2.0 ** -8 + 2.0 ** -18 * kr.abs().amax(-1, keepdim=True), torch.zeros_like(kr))):
                other = dst[0].clone()
                kv_layout.write_tokens(dst, torch.as_tensor(w.table[s]), one(a), one(b), pos)
                dst[0] = other                                   # (the other layer keeps what it had)
    got = w.cache.kv.cpu().double()
    assert bool(((got - want).abs() <= tol).all())
    if out_wide is not None and c["extra"]:
        assert bool((out_wide[:, :, :c["extra"]] == 7).all()) and bool((out_wide[:, :, -c["extra"]:] == 7).all())
    # the bounds of blocks that became whole are those of the cache as it is now
    ids = [int(w.table[s][b]) for s in range(n) for b in range(c["lens"][s] // 16, (c["lens"][s] + valid[s]) // 16) if valid[s]]
    if ids:
        lo, hi = w.cache.read_bounds(i32(ids))
        for j, b in enumerate(ids):
            tile = kv_layout._tiles_to_tokens_k(w.cache.kv[layer:layer + 1, 0, b:b + 1].cpu(), c["hd"])[0]
            for h in range(c["kv_heads"]):
                l, u = ref.bounds(tile[:, h])
                assert torch.equal(lo[layer, j, h].cpu().double(), l) and torch.equal(hi[layer, j, h].cpu().double(), u)


def test_append_skips_sequences_that_are_not_in_order():
    w = World([20, 20, 20, 20, 20], more=40)
    w.bt[1, 1] = w.cache.num_blocks                             # needed
    w.bt[2, 1] = -1                                             # needed
    w.bt[4, 0] = -5                                             # behind: not needed
    lens, valid = [20, 20, 20, -1, 20], [4, 4, 4, 4, 4]
    k, q = torch.randn(5, 4, 2, 64, device=DEV).to(torch.bfloat16), torch.randn(5, 4, 4, 64, device=DEV).to(torch.bfloat16)
    before, out, status = w.cache.kv.clone(), torch.full_like(q, 3.0), i32([9] * 5)
    w.cache.append(0, k, k, w.bt, i32(lens), q=q, q_out=out, n_valid=i32(valid), seq_status=status)
    assert status.tolist() == [0, 2, 2, 1, 0]
    assert torch.equal(out[[0, 4]], q[[0, 4]]) and bool((out[1:4] == 3).all())
    changed = (w.cache.kv != before).any(-1).any(-1).any(0).any(0).nonzero().flatten().tolist()
    assert sorted(changed) == sorted(int(w.table[s][1]) for s in (0, 4))
    w.cache.kv.copy_(before)
    for bad in ([5] * 5, [-1] * 5):
        w.cache.append(0, k, k, w.bt, i32(lens), q=q, q_out=out, n_valid=i32(bad), seq_status=status)
        assert status.tolist() == [1] * 5 and torch.equal(w.cache.kv, before)
    w.cache.append(0, k, k, w.bt, i32([20] * 5), q=q, q_out=out, max_context=23, seq_status=status)
    assert status.tolist() == [1] * 5 and torch.equal(w.cache.kv, before)


def test_far_positions_keep_their_angles():
    """Position 2^24 - 1: in fp32 its angle would be off by half a radian."""
    pos, rope = 2 ** 24 - 1, Rope(64, 1e4, 2 ** 24)
    kv = torch.zeros(1, 2, 1, 1, 16 * 64, dtype=torch.bfloat16, device=DEV)
    cache = PagedCache(kv, 1, 64, bounds=False)
    q = torch.randn(1, 1, 1, 64, device=DEV).to(torch.bfloat16)
    bt = torch.zeros(1, 2 ** 20, dtype=torch.int32, device=DEV)
    out = cache.append(0, q, q, bt, i32([pos]), q=q, rope=rope)
    want = ref.turned(q.cpu(), pos, None, 0, (64, 1e4, "half", dict(kind="none")))
    # (an angle near 2^24 in float64 is off by 2^-29: nothing here)
    assert bool(((out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + 2.0 ** -18 * want.abs().max()).all())


@pytest.mark.parametrize("hd,kv_heads", [(64, 1), (64, 3), (128, 2)])
def test_bounds_are_exact(hd, kv_heads):
    w = World([0, 15, 16, 17, 200], kv_heads, 1, hd)
    k = w.k[4]
    k[:, 0:16] = 0
    k[0, 20, 0, 3], k[0, 40, 0, 5], k[1, 60, -1, 7] = math.nan, -math.inf, math.inf
    k[0, 64:80] *= 2.0 ** 60                                     # beyond what has bounds
    k[0, 80:96] = 2.0 ** -100
    k[0, 96:112] = torch.randint(-3, 4, (16, kv_heads, hd), generator=w.g).to(torch.bfloat16) * 2.0 ** -41
    k[0, 112:128, :, 0] = 127 * 2.0 ** 40                        # the last that has
    k[0, 128:144] = 0
    k[0, 128:144, :, 1] = 254.0                                  # 127 * 2
    k[0, 128:144, :, 2] = -1.0
    k[0, 144:160, :, 1] = 255.0                                  # one more than that: 4 is the unit
    k[0, 160:176] = -0.0
    kv_layout.write_tokens(w.cache.kv, w.bt[4], k.to(DEV), w.v[4].to(DEV))
    w.cache.bounds.fill_(99)
    status = i32([7] * 5)
    w.cache.store_bounds(w.bt, i32([0, 0, 0, 0, 0]), i32(w.lens), 200, seq_status=status)
    assert status.tolist() == [0] * 5
    rec = w.cache.bounds.view(2, w.cache.num_blocks, kv_heads, 2 * hd + 16)
    done = set()
    for s, n in enumerate(w.lens):
        ids = [int(x) for x in w.table[s][:n // 16]]
        done |= set(ids)
        if not ids:
            continue
        lo, hi = w.cache.read_bounds(i32(ids))
        for layer in range(2):
            l, u = w.bounds(layer, s)
            assert torch.equal(lo[layer].cpu().double(), l) and torch.equal(hi[layer].cpu().double(), u), (s, layer)
    for b in range(w.cache.num_blocks):
        assert bool((rec[:, b] == 99).all()) == (b not in done)
    # a range that touches blocks 1 .. 4 and makes 1 .. 3 whole, in one layer
    w.cache.bounds.fill_(99)
    w.cache.store_bounds(w.bt[4:], i32([17]), i32([50]), 64, layer=1)
    touched = [int(x) for x in w.table[4][1:4]]
    assert sorted((rec != 99).any(-1).any(-1)[1].nonzero().flatten().tolist()) == sorted(touched) and bool((rec[0] == 99).all())
    # ids out of range leave zeros; flagged sequences nothing
    lo, hi = w.cache.read_bounds(i32([-1, w.cache.num_blocks, touched[0]]))
    assert bool((lo[:, :2] == 0).all()) and bool((hi[:, :2] == 0).all())
    assert w.cache.read_bounds(i32([]))[0].shape == (2, 0, kv_heads, hd)
    w.cache.bounds.fill_(99)
    table = w.bt[[4, 4, 4, 4]].clone()
    table[0, 2], table[1, 5] = -1, w.cache.num_blocks
    status = i32([7] * 4)
    w.cache.store_bounds(table, i32([32, 64, -1, 0]), i32([16, 32, 16, 65]), 64, seq_status=status)
    assert status.tolist() == [2, 2, 1, 1] and bool((w.cache.bounds == 99).all())
    w.cache.store_bounds(table, i32([32, 64, 300, 0]), i32([0, 15, 32, 0]), 64, seq_status=status)
    assert status.tolist() == [0, 0, 1, 0] and bool((w.cache.bounds == 99).all())


@pytest.mark.parametrize("hd", [64, 128])
def test_bounds_of_the_smallest_and_largest_keys(hd):
    """bf16 numbers below the normal ones still count, outward, as one unit of 2^-40; every border between two powers of two."""
    w = World([16 * 40], 1, 1, hd, layers=1)
    k = w.k[0]
    k[:] = 0
    k[0, 0:16, :, 0], k[0, 5, :, 1] = 2.0 ** -133, -(2.0 ** -130)
    for b in range(1, 40):
        e = 2 * b - 41
        k[0, 16 * b + 3, 0, b] = 127 * 2.0 ** e if b % 2 else 127.5 * 2.0 ** e
        k[0, 16 * b + 9, 0, b + 1] = -(2.0 ** (e - 3))
    kv_layout.write_tokens(w.cache.kv, w.bt[0], k.to(DEV), w.v[0].to(DEV))
    w.cache.store_bounds(w.bt, i32([0]), i32([640]), 640)
    lo, hi = w.cache.read_bounds(w.bt[0].contiguous())
    l, u = w.bounds(0, 0)
    assert torch.equal(lo[0].cpu().double(), l) and torch.equal(hi[0].cpu().double(), u)
    assert float(hi[0, 0, 0, 0]) == 2.0 ** -40 and float(lo[0, 0, 0, 1]) == -(2.0 ** -40)


def expected_lists(w, layer, q, lens, valid, budget, sink, recent):
    n, window = q.shape[:2]
    out = torch.full((n, window, w.kv_heads, budget), -77, dtype=torch.int32)
    for s in range(n):
        lo, hi = w.bounds(layer, s)
        for i in range(valid[s]):
            own = (lens[s] + i) // 16
            pad = lambda x: torch.cat([x, torch.zeros(max(0, own + 1 - len(x)), *x.shape[1:], dtype=x.dtype)])
            for h in range(w.kv_heads):
                qh = q[s, i, h * w.group:(h + 1) * w.group]
                out[s, i, h] = torch.tensor(ref.select(qh, pad(lo)[:, h], pad(hi)[:, h], own, budget, sink, recent), dtype=torch.int32)
    return out


SELECTS = [
    dict(lens=[600], budget=8), dict(lens=[0, 15, 16, 700, 333], budget=5, window=5, valid=[0, 5, 1, 4, 5], group=3),
    dict(lens=[500, 90], budget=16, window=13, group=4, hd=128, sink=0, recent=1), dict(lens=[1000], budget=3, sink=1, recent=2, group=1),
    dict(lens=[1000], budget=1, sink=0, recent=1), dict(lens=[1000], budget=2, sink=0, recent=1, group=16, kv_heads=1, window=3),
    dict(lens=[800], budget=64, sink=4, recent=8), dict(lens=[811, 799, 800, 801], budget=51, window=2, group=8), dict(lens=[640], budget=39, group=5, hd=128),
    dict(lens=[2500] * 3, budget=100, kv_heads=3, group=2, hd=128), dict(lens=[1300], budget=70, window=40, group=7, kv_heads=1),
]


@pytest.mark.parametrize("case", SELECTS, ids=lambda c: "-".join(str(v) for v in c.values()).replace(" ", ""))
@pytest.mark.parametrize("room", ["own", "longer"])
def test_select_is_exact(case, room):
    """`longer`: max_context as large as it takes for the scores to go through the workspace."""
    c = dict(window=1, kv_heads=2, group=2, hd=64, sink=1, recent=2, valid=None)
    c.update(case)
    w = World([n + c["window"] for n in c["lens"]], c["kv_heads"], c["group"], c["hd"])
    w.cache.store_bounds(w.bt, i32([0] * len(w.lens)), i32(w.lens), max(w.lens))
    q = w.queries(c["window"])
    valid = c["valid"] or [c["window"]] * len(w.lens)
    bt, most = w.bt, None
    if room == "longer":
        bt = torch.nn.functional.pad(w.bt, (0, 12289 * 16 - w.bt.shape[1]), value=-1)
        most = bt.shape[1] * 16
    out, status = torch.full((len(w.lens), c["window"], c["kv_heads"], c["budget"]), -77, dtype=torch.int32, device=DEV), i32([5] * len(w.lens))
    dq, _ = rows_in(q, 8, torch.bfloat16)
    w.cache.select(1, dq, bt, i32(c["lens"]), c["budget"], c["sink"], c["recent"], i32(valid) if c["valid"] else None, most, out, status)
    assert status.tolist() == [0] * len(w.lens)
    want = expected_lists(w, 1, q, c["lens"], valid, c["budget"], c["sink"], c["recent"])
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("blocks,window,group", [(1800, 3, 4), (5000, 1, 3), (9500, 2, 1), (1_100_000, 1, 2)])
def test_select_of_long_contexts(blocks, window, group):
    """Rows whose scores are held two or eight to a thread, or read again and again; more blocks than a launch has workgroups for 256 of them each."""
    hd, n = 64, blocks * 16
    g = torch.Generator(device=DEV).manual_seed(blocks)
    kv = torch.empty(1, 2, blocks, 1, 16 * hd, dtype=torch.bfloat16, device=DEV)
    kv[:, 0].normal_(generator=g)                                # (in whatever order: random is random)
    kv[0, 0, ::7] *= 1.5
    cache, table = PagedCache(kv, group, hd), torch.randperm(blocks, generator=g, device=DEV).int()[None]
    cache.store_bounds(table, i32([0]), i32([n]), n)
    lo, hi = (x[0, :, 0].cpu().double() for x in cache.read_bounds(table[0].contiguous()))
    q = torch.randn(1, window, group, hd, generator=g, device=DEV).to(torch.bfloat16)
    for budget, sink, recent in ((7, 1, 2), (130, 4, 8), (4096, 0, 1)):
        if budget < blocks:
            got = cache.select(0, q, table, i32([n - window]), budget, sink, recent)
            for i in range(window):
                assert got[0, i, 0].tolist() == ref.select(q[0, i].cpu(), lo, hi, (n - window + i) // 16, budget, sink, recent)


@pytest.mark.parametrize("room", ["own", "longer"])
def test_select_ties_and_values_without_an_order(room):
    w = World([1000] * 6, kv_heads=1, group=2, hd=64, layers=1)
    for s in range(6):
        if s != 1:
            w.k[s][0] = w.k[s][0, :16].repeat(63, 1, 1)[:1000]    # the same block again and again: all scores are equal
    w.k[1][0, 320] = math.nan                                     # blocks 20 and 40: infinite bounds
    w.k[1][0, 650, 0, 9] = math.inf
    w.k[2][0, 160:176] *= 4.0                                     # block 10: larger products of either sign
    q = w.queries(1)
    q[3, 0, 0, 5] = math.nan                                      # a head without an order counts as zeros, both: all ties
    q[3, 0, 1, 5] = math.inf
    q[4] = 0
    q[5, 0, 0] = 2.0 ** 100
    for s in range(6):
        kv_layout.write_tokens(w.cache.kv, w.bt[s], w.k[s].to(DEV), w.v[s].to(DEV))
    w.cache.store_bounds(w.bt, i32([0] * 6), i32(w.lens), 1000)
    bt = w.bt if room == "own" else torch.nn.functional.pad(w.bt, (0, 13000), value=-1)
    got = w.cache.select(0, q.to(DEV), bt, i32([990] * 6), 9, 2, 3)
    want = expected_lists(w, 0, q, [990] * 6, [1] * 6, 9, 2, 3)
    assert torch.equal(got.cpu(), want)
    assert want[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5, 59, 60, 61] and {20, 40} <= set(want[1, 0, 0].tolist()) and 10 in want[2, 0, 0]


@pytest.mark.parametrize("room", ["own", "longer"])
def test_select_skips_sequences_that_are_not_in_order(room):
    w = World([400] * 5)
    w.cache.store_bounds(w.bt, i32([0] * 5), i32(w.lens), 400)
    bt = w.bt.clone() if room == "own" else torch.nn.functional.pad(w.bt, (0, 13000), value=-1)
    bt[1, 0], bt[2, 24], bt[4, 13] = -1, w.cache.num_blocks, 2 ** 31 - 1
    out, status = torch.full((5, 2, 2, 8), -77, dtype=torch.int32, device=DEV), i32([9] * 5)
    w.cache.select(0, w.queries(2).to(DEV), bt, i32([398, 398, 398, -3, 100]), 8, selected=out, seq_status=status)
    assert status.tolist() == [0, 2, 2, 1, 0]
    assert bool((out[1:4] == -77).all()) and bool((out[[0, 4]] != -77).all())
    w.cache.select(0, w.queries(2).to(DEV), bt, i32([398] * 5), 8, n_valid=i32([3, 0, -1, 0, 2]), selected=out.fill_(-77), seq_status=status)
    assert status.tolist() == [1, 0, 1, 0, 2] and bool((out == -77).all())


def test_select_of_rows_that_are_not_there():
    """A window at the end of the room: its rows behind n_valid would see blocks that no array has."""
    w = World([16 * 800] * 2, kv_heads=1, group=1, hd=64, layers=1)
    w.cache.store_bounds(w.bt, i32([0] * 2), i32(w.lens), 12800)
    q, lens = w.queries(512), [12799, 12500]
    got = w.cache.select(0, q.to(DEV), w.bt, i32(lens), 6, n_valid=i32([1, 300]))
    few = [0, 1, 2, 17, 299]
    for s, rows in ((0, [0]), (1, few)):
        lo, hi = w.bounds(0, s)
        for i in rows:
            assert got[s, i, 0].tolist() == ref.select(q[s, i], lo[:, 0], hi[:, 0], (lens[s] + i) // 16, 6, 1, 2), (s, i)
    assert bool((got[0, 1:] == -1).all()) and bool((got[1, 300:] == -1).all())


def lists_of(w, lens, window, width, kind):
    """Lists of every kind, [seqs][window][kv heads][width]."""
    out = torch.full((len(lens), window, w.kv_heads, width), -1, dtype=torch.int32)
    for s, n in enumerate(lens):
        for i in range(window):
            own = (n + i) // 16
            for h in range(w.kv_heads):
                if kind == "ascending":
                    ids = sorted(torch.randperm(own, generator=w.g)[:width - 1].tolist()) + [own]
                elif kind == "mixed":                             # out of order, twice, beyond, below, holes
                    ids = torch.randint(-3, own + 4, (width,), generator=w.g).tolist()
                elif kind == "own":
                    ids = [-1] * (width - 1) + [own]
                else:
                    ids = []
                out[s, i, h, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    return out


ATTENDS = [
    dict(lens=[600]), dict(lens=[0, 15, 16, 300], window=5, valid=[5, 0, 1, 4], group=3, width=7), dict(lens=[500, 90], window=13, group=4, hd=128, width=16),
    dict(lens=[1000], group=16, kv_heads=1, hd=128, width=33), dict(lens=[1000, 3], width=1, hd=128), dict(lens=[1000, 1000], width=2, kind="mixed"),
    dict(lens=[700, 31, 700], window=3, width=37, kind="mixed", hd=128, group=8), dict(lens=[9000], width=600, hd=128, group=4),
    dict(lens=[9000, 200], width=513, kind="mixed", group=5, kv_heads=1), dict(lens=[300, 40], width=9, kind="own", hd=128),
    dict(lens=[300, 40], width=9, kind="none"), dict(lens=[5000], width=300, kind="none", hd=128), dict(lens=[5000] * 2, width=300, kind="own"),
    dict(lens=[100] * 40, window=8, width=4, group=1, kv_heads=3), dict(lens=[2000], width=128, hd=128, scale=0.25), dict(lens=[66000], width=4096, hd=64, kv_heads=1, group=1),
]


@pytest.mark.parametrize("case", ATTENDS, ids=lambda c: "-".join(str(v) for v in c.values()).replace(" ", ""))
def test_sparse_attention(case):
    c = dict(window=1, kv_heads=2, group=2, hd=64, valid=None, width=8, kind="ascending", scale=0.0)
    c.update(case)
    w = World([n + c["window"] for n in c["lens"]], c["kv_heads"], c["group"], c["hd"], layers=1, bounds=False)
    n, window = len(c["lens"]), c["window"]
    valid = c["valid"] or [window] * n
    q, lists = w.queries(window) * 0.7, lists_of(w, c["lens"], window, c["width"], c["kind"])
    # what no row may look at: positions behind the last row's, and blocks of nobody
    used = {int(x) for s in range(n) for x in w.table[s][:(w.lens[s] + 15) // 16]}
    poison = torch.tensor([b for b in range(w.cache.num_blocks) if b not in used], device=DEV)
    w.cache.kv[:, :, poison] = math.nan
    for s in range(n):
        end = c["lens"][s] + max(valid[s], 1)
        bad = torch.full((1, -end % 16, c["kv_heads"], c["hd"]), math.nan)
        if bad.shape[1]:
            kv_layout.write_tokens(w.cache.kv, w.bt[s], bad.to(DEV), bad.to(DEV), end)
    (dq, _), (out, wide) = rows_in(q, 8, torch.bfloat16), rows_in(torch.full(q.shape, 9.0), 16, torch.bfloat16)
    status = i32([4] * n)
    got = w.cache.attention(0, dq, w.bt, i32(c["lens"]), lists.to(DEV), i32(valid) if c["valid"] else None, out=out, scale=c["scale"], seq_status=status)
    assert got is out and status.tolist() == [0] * n
    assert bool((wide[:, :, :16] == 7).all()) and bool((wide[:, :, -16:] == 7).all())
    scale = c["scale"] or c["hd"] ** -0.5
    for s in range(n):
        assert bool((out[s, valid[s]:] == 9).all())
        for i in range(valid[s]):
            for h in range(c["kv_heads"]):
                mine = slice(h * c["group"], (h + 1) * c["group"])
                o, mag = ref.attention(q[s, i, mine], w.k[s][0, :, h], w.v[s][0, :, h], lists[s, i, h].tolist(), c["lens"][s] + i, scale)
                assert bool(((out[s, i, mine].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2.0 ** -12 * mag).all()), (s, i, h)


@pytest.mark.parametrize("width", [6, 300])
def test_sparse_attention_leaves_rows_with_bad_blocks(width):
    w = World([400] * 4, layers=1, bounds=False)
    lists = torch.full((4, 2, 2, width), -1, dtype=torch.int32)
    lists[..., -1] = 3
    lists[..., 0] = torch.tensor([1, 2])                          # kv head 0 reads block 1, 1 reads 2
    bt = w.bt.clone()
    bt[1, 1] = -1
    bt[2, 7] = w.cache.num_blocks                                 # listed by nobody
    q = w.queries(2).to(DEV)
    out, status = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV), i32([4] * 4)
    w.cache.attention(0, q, bt, i32([390, 390, 390, 500]), lists.to(DEV), out=out, seq_status=status)
    assert status.tolist() == [0, 2, 0, 1]
    want = w.cache.attention(0, q, w.bt, i32([390] * 4), lists.to(DEV))
    assert torch.equal(out[[0, 2]], want[[0, 2]]) and torch.equal(out[1, :, 2:], want[1, :, 2:])
    assert bool((out[1, :, :2] == 9).all()) and bool((out[3] == 9).all())


def test_infinities_and_nan_are_those_of_the_softmax():
    w = World([64] * 3, kv_heads=1, group=1, layers=1, bounds=False)
    w.k[0][0, 5, 0, 0], w.v[1][0, 7, 0, 3], w.k[2][0, 9, 0, 0] = math.nan, math.inf, -math.inf
    for s in range(3):
        kv_layout.write_tokens(w.cache.kv, w.bt[s], w.k[s].to(DEV), w.v[s].to(DEV))
    q = w.queries(1)
    q[:, :, :, 0] = 1.0
    lists = torch.tensor([0, 1], dtype=torch.int32).expand(3, 1, 1, 2).contiguous()
    out = w.cache.attention(0, q.to(DEV), w.bt, i32([63] * 3), lists.to(DEV)).cpu()
    assert bool(torch.isnan(out[0]).all())
    assert math.isinf(out[1, 0, 0, 3]) and int(torch.isfinite(out[1]).sum()) == 63
    o, mag = ref.attention(q[2, 0], w.k[2][0, :, 0], w.v[2][0, :, 0], [0, 1], 63, 0.125)      # one key with a weight of 0
    assert bool(((out[2, 0].double() - o).abs() <= o.abs() * 2.0 ** -8 + 2.0 ** -12 * mag).all())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("pos", [0, 5, 40])
def test_infinite_values_stay_infinite(hd, pos):
    """Whatever their weights are, 1 among them (the only key, or one of equal keys)."""
    w = World([64], kv_heads=2, group=4, hd=hd, layers=1, bounds=False)
    w.k[0][:] = 0
    w.v[0][0, 0, :, 1], w.v[0][0, 0, :, 2] = math.inf, -math.inf
    kv_layout.write_tokens(w.cache.kv, w.bt[0], w.k[0].to(DEV), w.v[0].to(DEV))
    lists = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV).expand(1, 1, 2, 3).contiguous()
    out = w.cache.attention(0, w.queries(1).to(DEV), w.bt, i32([pos]), lists).cpu()
    assert bool((out[..., 1] == math.inf).all()) and bool((out[..., 2] == -math.inf).all())
    want = w.v[0][0, :pos + 1].double().mean(0).repeat_interleave(4, 0)
    fine = torch.tensor([f for f in range(hd) if f not in (1, 2)])
    assert bool(((out[0, 0][:, fine].double() - want[:, fine]).abs() <= want[:, fine].abs() * 2.0 ** -8 + 2.0 ** -12 * w.v[0][0, :pos + 1].double().abs().mean(0).repeat_interleave(4, 0)[:, fine]).all())


def test_offsets_beyond_32_bits():
    """Blocks whose keys, values and bounds lie 2^32 bytes and 2^31 elements behind their arrays' beginnings."""
    h, hd, blocks = 8, 128, 2_100_000                             # K plane: 34.4e9 elements; bounds: 4.57e9 bytes
    heads, width = B.Heads(1, h, h, hd), 40
    kv = torch.empty((1, 2, blocks, h, 16 * hd), dtype=torch.bfloat16, device=DEV)
    cache = PagedCache(kv, h, hd)
    ids = torch.arange(blocks - width, blocks, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(1, 624, h, hd, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    small = PagedCache(torch.zeros((1, 2, width, h, 16 * hd), dtype=torch.bfloat16, device=DEV), h, hd)
    near = torch.arange(width, dtype=torch.int32, device=DEV)[None].contiguous()
    got = []
    for c, bt in ((cache, ids), (small, near)):
        rope = Rope(hd, 1e4, 640)
        for at in (0, 312):
            q = c.append(0, k[:, at:at + 312], v[:, at:at + 312], bt, i32([at]), q=k[:, at:at + 312], rope=rope)
        lists = c.select(0, q[:, -2:], bt, i32([622]), 12)
        got.append((lists, c.attention(0, q[:, -2:], bt, i32([622]), lists)) + c.read_bounds(bt[0, :39].contiguous()))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    del kv, cache


def test_the_most_rows_of_a_call():
    """65536 sequences of a token each: append, bounds, selection and attention, looked at in some of them and by their sums in all."""
    n, hd, blocks = 65536, 64, 3
    g = torch.Generator(device=DEV).manual_seed(5)
    table = torch.randperm(n * blocks, generator=g, device=DEV).int().view(n, blocks)
    k, v = (torch.randn(n, blocks * 16, 1, hd, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    kv = torch.zeros(1, 2, n * blocks, 1, 16 * hd, dtype=torch.bfloat16, device=DEV)
    at = table.flatten().long()
    kv[0, 0, at] = kv_layout._tokens_to_tiles_k(k.view(1, -1, 1, hd), hd)[0]
    kv[0, 1, at] = kv_layout._tokens_to_tiles_v(v.view(1, -1, 1, hd), hd)[0]
    cache, lens = PagedCache(kv, 2, hd), torch.randint(0, 47, (n,), generator=g, device=DEV).int()
    lens[:3] = torch.tensor([0, 15, 46])
    start = kv.clone()
    cache.store_bounds(table, torch.zeros_like(lens), lens, 48)
    q, nk, nv = (torch.randn(n, 1, h, hd, generator=g, device=DEV).to(torch.bfloat16) for h in (2, 1, 1))
    rope, status = Rope(hd, 1e4, 64), torch.full((n,), 9, dtype=torch.int32, device=DEV)
    turned = cache.append(0, nk, nv, table, lens, q=q, rope=rope, seq_status=status)
    assert int(status.abs().sum()) == 0
    lists = cache.select(0, turned, table, lens, 2, 0, 1, seq_status=status.fill_(9))
    assert int(status.abs().sum()) == 0
    out = cache.attention(0, turned, table, lens, lists, seq_status=status.fill_(9))
    assert int(status.abs().sum()) == 0
    own = (lens // 16)[:, None, None]
    assert bool((lists[..., 0] <= own).all()) and bool((torch.where(own > 0, lists[..., 1], lists[..., 0]) == own).all())
    # one position of every sequence has changed, in K and in V
    read = lambda c: (kv_layout._tiles_to_tokens_k(c[:, 0, at], hd)[0].view(n, 48, hd), kv_layout._tiles_to_tokens_v(c[:, 1, at], hd)[0].view(n, 48, hd))
    (k0, v0), (k1, v1) = read(start), read(kv)
    here = torch.arange(48, device=DEV) == lens[:, None]
    assert torch.equal(v1, torch.where(here[..., None], nv.view(n, 1, hd), v0)) and torch.equal(k1[~here], k0[~here])
    for s in [0, 1, 2, 3, 1000, 32767, 32768, 65535] + [int(x) for x in torch.randint(0, n, (60,), generator=g, device=DEV)]:
        pos = int(lens[s])
        ks, vs = k1[s].cpu(), v1[s].cpu()
        for got, plain in ((turned[s, 0], q[s, 0]), (ks[pos:pos + 1], nk[s, 0])):
            want = ref.turned(plain.cpu(), pos, None, 0, (hd, 1e4, "half", dict(kind="none")))
            assert bool(((got.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + 2.0 ** -18 * want.abs().max()).all())
        pairs = [ref.bounds(ks[16 * b:16 * b + 16]) for b in range(pos // 16 + 1)]
        lo, hi = (torch.stack([x[i] for x in pairs]) for i in range(2))
        assert lists[s, 0, 0].tolist() == ref.select(turned[s, 0].cpu(), lo, hi, pos // 16, 2, 0, 1)
        o, mag = ref.attention(turned[s, 0].cpu(), ks, vs, lists[s, 0, 0].tolist(), pos, 0.125)
        assert bool(((out[s, 0].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2.0 ** -12 * mag).all())


@pytest.mark.parametrize("hd,group", [(64, 2), (128, 4)])
def test_a_layer_by_the_operators(hd, group):
    """Prompts appended in windows, then tokens one by one: where the budget covers the context, attention is the dense one; where it does not,
    it is that over the selected blocks."""
    kv_heads, lens, layer = 2, [70, 131], 1
    w = World([0, 0], kv_heads, group, hd, more=200)
    rope_is = (hd, 1e4, "half", LLAMA3)
    rope = Rope(hd, 1e4, 256, "half", LLAMA3)
    gains = [(1 + 0.1 * torch.randn(hd, generator=w.g)).to(torch.bfloat16) for _ in range(2)]
    q, k, v = (torch.randn(2, 160, h, hd, generator=w.g).to(torch.bfloat16) for h in (kv_heads * group, kv_heads, kv_heads))
    keys = torch.stack([torch.stack([ref.turned(k[s, p], p, gains[1], 1e-6, rope_is) for p in range(160)]) for s in range(2)])
    done, step = [0, 0], 0
    while max(done) < 158:
        window = 48 if step < 3 else 1
        n = [min(window, max(0, lens[s] - done[s])) if step < 3 else 1 for s in range(2)]
        take = lambda x: torch.stack([torch.nn.functional.pad(x[s, done[s]:done[s] + window], (0, 0, 0, 0, 0, window - len(x[s, done[s]:done[s] + window])))
                                      for s in range(2)]).to(DEV)
        at = i32(done)
        turned = w.cache.append(layer, take(k), take(v), w.bt, at, q=take(q), n_valid=i32(n), rope=rope, q_norm=gains[0].to(DEV), k_norm=gains[1].to(DEV))
        check = step < 3 or done[0] % 13 == 0
        for budget in (16, 4) if check else ():
            lists = w.cache.select(layer, turned, w.bt, at, budget, n_valid=i32(n))
            out = w.cache.attention(layer, turned, w.bt, at, lists, n_valid=i32(n))
            for s in range(2):
                for i in range(0, n[s], 11):
                    for h in range(kv_heads):
                        blocks = lists[s, i, h].tolist()
                        pos = done[s] + i
                        assert pos // 16 in blocks and (budget < 16 or [b for b in blocks if b >= 0] == list(range(pos // 16 + 1)))
                        qq = ref.turned(q[s, pos, h * group:(h + 1) * group], pos, gains[0], 1e-6, rope_is)
                        o, mag = ref.attention(qq, keys[s, :, h], v[s, :, h], blocks, pos, hd ** -0.5)
                        # q and the keys are held in bf16: a score is off by 2^-7 of sum |q k| / sqrt(hd) <= |q| |k| 2^-7 / sqrt(hd) at the worst
                        worst = float((qq.norm(dim=-1).max() * keys[s, :pos + 1, h].norm(dim=-1).max()) * hd ** -0.5) * 2.0 ** -7
                        lim = o.abs() * 2.0 ** -8 + mag * (2.0 ** -12 + 2 * math.expm1(worst))
                        assert bool(((out[s, i, h * group:(h + 1) * group].cpu().double() - o).abs() <= lim).all())
        done = [done[s] + n[s] for s in range(2)]
        step += 1


def test_graph_replays_follow_their_inputs():
    w = World([1500] * 3, kv_heads=2, group=4, hd=128, layers=1, more=64)
    w.cache.store_bounds(w.bt, i32([0] * 3), i32(w.lens), 1500)
    rope, start = Rope(128, 1e4, 2048), w.cache.kv.clone()
    rows = torch.zeros(3, 1, 12 * 128, dtype=torch.bfloat16, device=DEV)
    q, k, v = (x.unflatten(-1, (-1, 128)) for x in rows.split([8 * 128, 2 * 128, 2 * 128], -1))
    lens = i32(w.lens)

    def step():
        turned = w.cache.append(0, k, v, w.bt, lens, q=q, rope=rope)
        lists = w.cache.select(0, turned, w.bt, lens, 300 if wide else 24)
        return lists, w.cache.attention(0, turned, w.bt, lens, lists)

    for wide in (False, True):                                    # (lists of 300 are attended to in parts)
        w.cache.kv.copy_(start)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lists, out = step()
        g = torch.Generator(device=DEV).manual_seed(1)
        for turn in range(4):
            rows.copy_(torch.randn(rows.shape, generator=g, device=DEV))
            w.cache.kv.copy_(start)
            graph.replay()
            torch.cuda.synchronize()
            got = lists.clone(), out.clone(), w.cache.kv.clone()
            w.cache.kv.copy_(start)
            want = step()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], w.cache.kv)
            lens += 1
        lens.copy_(i32(w.lens))


def test_calls_on_two_streams_share_nothing():
    w = World([3000] * 8, kv_heads=2, group=4, hd=128, layers=1)
    w.cache.store_bounds(w.bt, i32([0] * 8), i32(w.lens), 3000)
    lens = i32([2999] * 8)
    bt = torch.nn.functional.pad(w.bt, (0, 13000), value=-1)     # (scores through the workspace, lists of 300 in parts)
    q = [w.queries(1).to(DEV) for _ in range(2)]
    call = lambda x: w.cache.attention(0, x, bt, lens, w.cache.select(0, x, bt, lens, 150))
    want = [call(x) for x in q]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                got[j].append(call(q[j]))
    torch.cuda.synchronize()
    for j in range(2):
        assert all(torch.equal(x, want[j]) for x in got[j])


def test_python_refusals():
    w = World([100], bounds=False)
    q, k = w.queries(1).to(DEV), torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    lens = i32([50])
    lists = torch.zeros(1, 1, 2, 4, dtype=torch.int32, device=DEV)
    rope, narrow = Rope(128, 1e4, 64), Rope(64, 1e4, 32)
    for call in (lambda: w.cache.select(0, q, w.bt, lens, 4), lambda: w.cache.store_bounds(w.bt, lens, lens, 4), lambda: w.cache.read_bounds(lens),
                 lambda: w.cache.attention(0, q.float(), w.bt, lens, lists), lambda: w.cache.attention(0, q[..., :32], w.bt, lens, lists),
                 lambda: w.cache.attention(0, q, w.bt, lens, lists.long()), lambda: w.cache.attention(0, q, w.bt, lens, lists[:, :, :1]),
                 lambda: w.cache.attention(0, q.cpu(), w.bt, lens, lists), lambda: w.cache.attention(0, q, w.bt[:, ::2], lens, lists),
                 lambda: w.cache.append(0, k, k.float(), w.bt, lens), lambda: w.cache.append(0, k, k, w.bt, lens, q=k),
                 lambda: w.cache.append(0, k.half(), k.half(), w.bt, lens), lambda: w.cache.append(0, k, k, w.bt, lens, k_norm=k[0, 0, 0, :32]),
                 lambda: w.cache.append(0, k.transpose(2, 3).contiguous().transpose(2, 3), k, w.bt, lens),
                 lambda: PagedCache(w.cache.kv.float(), 4, 64), lambda: PagedCache(w.cache.kv, 4, 128),
                 lambda: Rope(64, 1e4, 10, layout="both"), lambda: Rope(64, 1e4, 10, scaling=dict(kind="ntk")),
                 lambda: Rope(64, 1e4, 10, scaling=dict(kind="linear")), lambda: Rope(64, 1e4, 10, scaling=dict(kind="none", factor=2.0)),
                 lambda: PagedCache(w.cache.kv, 4, 64, bounds=torch.zeros(8, dtype=torch.uint8, device=DEV)).select(0, q, w.bt, lens, 4)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: w.cache.append(0, k, k, w.bt, lens, rope=rope), B.LLM42_EINVAL), (lambda: w.cache.append(2, k, k, w.bt, lens), B.LLM42_EINVAL),
                       (lambda: w.cache.append(0, k, k, w.bt, lens, rope=narrow, max_context=33), B.LLM42_ECAPACITY),
                       (lambda: PagedCache(w.cache.kv, 5, 64), B.LLM42_ESHAPE), (lambda: Rope(63, 1e4, 10), B.LLM42_EINVAL),
                       (lambda: w.cache.attention(0, q, w.bt, lens, lists, max_context=w.bt.shape[1] * 16 + 1), B.LLM42_ECAPACITY)):
        with pytest.raises(B.Llm42Error) as e:
            call()
        assert e.value.status == code
