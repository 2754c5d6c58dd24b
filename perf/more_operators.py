"""The operators around the paged bf16 cache, as cases that can be timed and compared with their plain forms.

  append     rows of new tokens: a norm for each head of Q and K, the rotation to their positions, K and V into the cache
  bounds     the 8-bit bounds of every block of 16 cached keys, and what they stand for
  select     the blocks that a query reads: the first ones, the last ones, and those whose keys may give the largest scores
  attention  of the new tokens over the blocks that were selected for them

Bounds of a block and kv head: 2^e is the smallest power of two (e at least -40) with every |key| <= 127 * 2^e; for each feature the
largest key is rounded up and the smallest down to whole multiples of it.  A query head is rounded to whole multiples of such a power of its own (ties
to even).  A block's score is the largest, over the query heads of the kv head, of the sum over the features of the larger of the products
of the query with the two bounds.  Products and sums are whole numbers below 2^24 times a power of two: exact in fp32, in any order.

A case's lengths follow from the case alone, so that every seed of it costs the same.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DEVICE = "cuda:0"
BLOCK = 16
EPS = 1e-6
PLAIN = dict(kind="none")
BANDS = dict(kind="llama3", factor=8.0, low_freq_factor=1.0, high_freq_factor=4.0, original_max_position=8192)
RAMP = dict(kind="yarn", factor=4.0, beta_fast=32.0, beta_slow=1.0, original_max_position=32768)
SCALINGS = {"none": PLAIN, "linear": dict(kind="linear", factor=4.0), "llama3": BANDS, "yarn": RAMP}


def _append(name, **kw):
    case = dict(name=name, op="append", seqs=1, window=1, kv_heads=8, group=4, hd=128, lo=0, hi=0, ragged=False, type="bf16", rot=128,
                layout="half", scaling="none", theta=5e5, norms=False, kept=1 << 30)
    case.update(kw)
    return case


def listed():
    return [
        # The token of a single interactive request: launch and latency only.
        _append("append_1x1", lo=511, hi=511),
        # Windows of a few tokens, partly filled, straight from fp32 sums, with the small test model's heads and half of each rotated.
        _append("append_5x13_hd64", seqs=5, window=13, kv_heads=2, group=2, hd=64, lo=0, hi=1900, ragged=True, type="f32", rot=32,
                layout="interleaved", scaling="linear", theta=1e4, norms=True),
        # A decode step of a full server, with normed heads and frequencies rescaled in bands (of the positions behind, which the call
        # does not touch, only the last blocks are there).
        _append("append_128x1", seqs=128, lo=1023, hi=8191, scaling="llama3", norms=True, kept=64),
        # A pass of long prompts far into their contexts.
        _append("append_8x512", seqs=8, window=512, lo=1000, hi=120000, scaling="yarn", theta=1e6, norms=True, kept=64),
        # What verified windows add to the bounds, all layers.
        dict(name="bounds_24x32", op="bounds", layers=32, seqs=24, kv_heads=8, hd=128, first_hi=400, lo=1, hi=32),
        # Prompts that have been prefilled, all layers.
        dict(name="bounds_4x2048", op="bounds", layers=32, seqs=4, kv_heads=8, hd=128, first_hi=0, lo=1500, hi=2048),
        # Blocks for windows of a few tokens, partly filled, with the small test model's heads ...
        dict(name="select_5x13_hd64", op="select", seqs=5, window=13, kv_heads=2, group=2, hd=64, lo=0, hi=1900, ragged=True, budget=16,
             sink=1, recent=2),
        # ... for a decode step of a full server with long contexts ...
        dict(name="select_128x8192", op="select", seqs=128, window=1, kv_heads=8, group=4, hd=128, lo=1023, hi=8191, ragged=False, budget=64,
             sink=1, recent=2),
        # ... and for one request behind a very long document.
        dict(name="select_1x131072", op="select", seqs=1, window=1, kv_heads=8, group=4, hd=128, lo=131071, hi=131071, ragged=False,
             budget=128, sink=4, recent=8),
        # Attention over them: a single interactive request ...
        dict(name="attention_1x64", op="attention", seqs=1, window=1, kv_heads=8, group=4, hd=128, lo=8191, hi=8191, ragged=False, budget=64),
        # ... windows of a few tokens, partly filled, with the small test model's heads ...
        dict(name="attention_5x13_hd64", op="attention", seqs=5, window=13, kv_heads=2, group=2, hd=64, lo=0, hi=1900, ragged=True,
             budget=16),
        # ... and a decode step of a full server.
        dict(name="attention_128x64", op="attention", seqs=128, window=1, kv_heads=8, group=4, hd=128, lo=1023, hi=8191, ragged=False,
             budget=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "bounds", "select", "select", "attention", "attention", "attention"])
    kv_heads, hd = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128])
    if op == "bounds":
        layers, seqs = rng.choice([1, 2, 4, 32]), _log_int(rng, 1, 64)
        most = 32 * 4 * 2048 * 8 * 128 // (layers * seqs * kv_heads * hd)
        hi = _log_int(rng, 16, min(2048, most))
        return dict(op=op, layers=layers, seqs=seqs, kv_heads=kv_heads, hd=hd, first_hi=min(rng.choice([0, 15, 400, 2000]), max(0, most - hi)),
                    lo=rng.randint(0, hi), hi=hi)
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
    window = rng.choice([1, 1, 1, 2, 3, 5, 8, 16, 32, _log_int(rng, 1, 64)])
    ragged = rng.random() < 0.5
    heads = kv_heads * group * hd
    if op == "append":
        if rng.random() < 0.3:
            window = _log_int(rng, 64, 512)
        seqs = _log_int(rng, 1, max(1, min(128, 8 * 512 * 32 * 128 // (window * (heads + 2 * kv_heads * hd)))))
        hi = _log_int(rng, 1, 30000)
        scaling = rng.choice(["none", "linear", "llama3", "yarn"])
        rot = rng.choice([hd, hd, hd // 2, hd // 4, 2 * rng.randint(1, hd // 2)]) if scaling != "yarn" else rng.choice([hd, hd // 2])
        case = _append("", seqs=seqs, window=window, kv_heads=kv_heads, group=group, hd=hd, lo=rng.randint(0, hi), hi=hi, ragged=ragged,
                       type=rng.choice(["bf16", "f32"]), rot=rot, layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                       theta=rng.choice([1e4, 5e5, 1e6]), norms=rng.random() < 0.5, kept=64)
        del case["name"]
        return case
    seqs = _log_int(rng, 1, 128)
    if op == "select":                               # some rows at least have more blocks than they may read
        cost = window * max(kv_heads * group, 8)
        seqs = max(1, min(seqs, 128 * 4608 * 8 * 4 // (cost * 500)))
        hi = _log_int(rng, 500, min(131071, 128 * 4608 * 8 * 4 // (seqs * cost), 128 * 8192 // seqs))
        budget = _log_int(rng, 2, min(128, hi // BLOCK // 2))
        sink = rng.randint(0, min(4, budget - 2))
        return dict(op=op, seqs=seqs, window=window, kv_heads=kv_heads, group=group, hd=hd, lo=rng.randint(0, hi), hi=hi, ragged=ragged,
                    budget=budget, sink=sink, recent=rng.randint(1, min(8, budget - sink - 1)))
    room = 128 * 64 * 8 * 128 * 4 // (window * kv_heads * hd * max(group, 4))
    budget = _log_int(rng, 1, min(128, room))
    seqs = min(seqs, room // budget)
    hi = _log_int(rng, 1, max(1, min(32000, 128 * 4608 // seqs)))
    return dict(op=op, seqs=seqs, window=window, kv_heads=kv_heads, group=group, hd=hd, lo=rng.randint(0, hi), hi=hi, ragged=ragged,
                budget=budget)


def _lengths(case):
    """(first or cached length, count or valid rows) of every sequence: a function of the case alone."""
    r = np.random.Generator(np.random.PCG64([case["seqs"], case["kv_heads"], case["hd"], case["lo"], case["hi"]]))
    n = case["seqs"]
    if case["op"] == "bounds":
        count = r.integers(case["lo"], case["hi"] + 1, n)
        count[0] = case["hi"]
        return r.integers(0, case["first_hi"] + 1, n), count
    cached = r.integers(case["lo"], case["hi"] + 1, n)
    cached[0] = case["hi"]
    valid = r.integers(0, case["window"] + 1, n) if case["ragged"] else np.full(n, case["window"])
    valid[0] = case["window"]
    return cached, valid


def work(case):
    a, b = _lengths(case)
    if case["op"] == "bounds":                       # every block that is whole and was touched: keys read, bounds written and read, values written
        blocks = int(np.maximum((a + b) // BLOCK - a // BLOCK, 0).sum()) * case["layers"] * case["kv_heads"]
        return {"bytes": blocks * case["hd"] * (2 * BLOCK + 2 * 2 + 2 * 2), "flops": blocks * case["hd"] * 2 * BLOCK}
    row, rows = case["kv_heads"] * case["hd"], int(b.sum())
    q = row * case["group"]
    if case["op"] == "append":
        values = rows * (q + 2 * row)
        return {"bytes": values * (TYPES[case["type"]].itemsize + 2) + rows * case["rot"] * 4, "flops": rows * (q + row) * 8}
    seen = _seen_blocks(case)
    if case["op"] == "select":                       # queries and the bounds of every block read, lists written
        blocks = int(((a + b) // BLOCK)[b > 0].sum())
        return {"bytes": 2 * rows * q + blocks * 2 * row + 4 * rows * case["kv_heads"] * case["budget"],
                "flops": 4 * int(seen.sum()) * q}
    listed_blocks = int(np.minimum(seen, case["budget"]).sum())
    return {"bytes": 4 * rows * q + listed_blocks * row * BLOCK * 2 * 2 + 4 * listed_blocks * case["kv_heads"],
            "flops": 4 * listed_blocks * BLOCK * q}


def _seen_blocks(case):
    """Blocks that each row sees, its own among them."""
    a, b = _lengths(case)
    return np.concatenate([(s + np.arange(n)) // BLOCK + 1 for s, n in zip(a, b)] or [np.zeros(0, np.int64)])


# ---- inputs ---------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _i32(x):
    return torch.as_tensor(np.asarray(x).astype(np.int32), device=DEVICE)


def _table(blocks_of, seed):
    """Blocks of every sequence, in no order and with three spare ones; entries that are not needed are -1."""
    total = int(blocks_of.sum())
    ids = np.random.Generator(np.random.PCG64([seed, 3])).permutation(total + 3)[:total]
    table = np.full((len(blocks_of), max(1, int(blocks_of.max()))), -1, np.int32)
    table[np.arange(table.shape[1]) < blocks_of[:, None]] = ids
    return table, total + 3


def _keys(g, shape, kv_heads, hd):
    """Keys, channels of different size, as rotary embeddings leave them; shape ends in kv_heads, hd."""
    k = torch.randn(shape, generator=g, device=DEVICE)
    return (k * (0.3 + 2.0 * torch.rand(kv_heads, hd, generator=g, device=DEVICE))).to(torch.bfloat16)


def _tiles(k, v):
    """Blocks of 16 tokens [..., 16, kv_heads, hd] in the cache's order [..., kv_heads, 16 * hd]."""
    lead, (h, hd) = k.shape[:-3], k.shape[-2:]
    n = len(lead)
    k = k.reshape(*lead, 16, h, hd // 8, 8).permute(*range(n), n + 1, n + 2, n, n + 3)
    v = v.reshape(*lead, 4, 4, h, hd // 16, 16).permute(*range(n), n + 2, n + 3, n, n + 4, n + 1)
    return k.reshape(*lead, h, 16 * hd), v.reshape(*lead, h, 16 * hd)


def _paged(k, v, table, blocks):
    """The cache [layers, 2, blocks, kv_heads, 16 * hd] that holds k, v [layers, seqs, tokens, kv_heads, hd] (tokens a multiple of 16)."""
    layers, seqs, tokens, h, hd = k.shape
    kv = torch.zeros((layers, 2, blocks, h, 16 * hd), dtype=torch.bfloat16, device=DEVICE)
    bt = torch.as_tensor(table[:, :tokens // 16], device=DEVICE).long()
    there = bt >= 0
    for i in range(layers):
        for plane, tiles in enumerate(_tiles(k[i].reshape(seqs, tokens // 16, 16, h, hd), v[i].reshape(seqs, tokens // 16, 16, h, hd))):
            kv[i, plane, bt[there]] = tiles[there]
    return kv


def _append_inputs(case, seed):
    g = _generator(seed)
    a, b = _lengths(case)
    h, hd, n, w = case["kv_heads"], case["hd"], case["seqs"], case["window"]
    # the blocks near the end of every sequence, and a table in which whatever is behind them shares the block 0
    needed = (a + b + BLOCK - 1) // BLOCK
    keep = np.minimum(needed, (case["kept"] + w) // BLOCK + 2)
    near, blocks = _table(keep, seed)
    table = np.zeros((n, max(1, int(needed.max()))), np.int32)
    for s in range(n):
        table[s, needed[s] - keep[s]:needed[s]] = near[s, :keep[s]] + 1
    kv = torch.randn((1, 2, blocks + 1, h, 16 * hd), generator=g, device=DEVICE).to(torch.bfloat16)
    # one matrix product gives q, k and v: they lie side by side in its rows
    rows = torch.randn((n, w, (case["group"] + 2) * h * hd), generator=g, device=DEVICE)
    rows = (rows * (0.3 + 2.0 * torch.rand(rows.shape[-1], generator=g, device=DEVICE))).to(TYPES[case["type"]])
    q, k, v = (x.unflatten(-1, (-1, hd)) for x in rows.split([case["group"] * h * hd, h * hd, h * hd], -1))
    norms = [(1.0 + 0.2 * torch.randn(hd, generator=g, device=DEVICE)).to(torch.bfloat16) if case["norms"] else None for _ in range(2)]
    return q, k, v, norms, kv, table


def _context(case, seed, values=True):
    """K and V [1, seqs, tokens, kv_heads, hd], tokens up to the next block's end of the longest sequence."""
    g = _generator(seed)
    a, b = _lengths(case)
    tokens = (int((a + b).max()) + BLOCK - 1) // BLOCK * BLOCK
    shape = (1, case["seqs"], tokens, case["kv_heads"], case["hd"])
    k = _keys(g, shape, case["kv_heads"], case["hd"])
    v = torch.randn(shape, generator=g, device=DEVICE).to(torch.bfloat16) if values else None
    q = torch.randn((case["seqs"], case["window"], case["kv_heads"] * case["group"], case["hd"]), generator=g, device=DEVICE)
    return k, v, q.to(torch.bfloat16), g


def _random_lists(case, g):
    """For every row and kv head `budget` of the blocks that it sees, its own among them, ascending, -1 behind them; the same blocks
    for all rows that see less than that."""
    a, b = _lengths(case)
    own_block = (_i32(a)[:, None] + torch.arange(case["window"], device=DEVICE)) // BLOCK                 # [seq][row]
    blocks = int((a + case["window"]).max()) // BLOCK + 1
    budget = case["budget"]
    out = torch.full((case["seqs"], case["window"], case["kv_heads"], budget), -1, dtype=torch.int32, device=DEVICE)
    at = torch.arange(blocks, device=DEVICE)
    for s in range(case["seqs"]):
        own_ = own_block[s, :, None, None]
        key = torch.rand((case["window"], case["kv_heads"], blocks), generator=g, device=DEVICE)
        key = key.masked_fill(at == own_, 2.0).masked_fill(at > own_, -1.0)
        best, ids = key.topk(min(budget, blocks), -1)
        ids = ids.masked_fill(best < 0, blocks).sort(-1).values
        out[s, :, :, :ids.shape[-1]] = torch.where(ids == blocks, -1, ids).int()
    return out


def _bounds_inputs(case, seed):
    g = _generator(seed)
    a, b = _lengths(case)
    tokens = (int((a + b).max()) + BLOCK - 1) // BLOCK * BLOCK
    return _keys(g, (case["layers"], case["seqs"], max(tokens, BLOCK), case["kv_heads"], case["hd"]), case["kv_heads"], case["hd"])


def _touched(case):
    """(sequence, block) of every block that is whole behind the call and holds one of its positions."""
    a, b = _lengths(case)
    return [(s, x) for s, (f, n) in enumerate(zip(a, b)) if n for x in range(f // BLOCK, (f + n) // BLOCK)]


def _cache(case, kv, bounds):
    from paper_2601_17768_amd.paged import PagedCache
    return PagedCache(kv, case["kv_heads"] * case.get("group", 1), case["hd"], bounds=bounds)


def prepare(case, seed):
    st = dict(case=case)
    a, b = _lengths(case)
    if case["op"] == "append":
        st["q"], st["k"], st["v"], st["norms"], st["kv"], table = _append_inputs(case, seed)
        st["bt"], st["lens"], st["valid"] = torch.as_tensor(table, device=DEVICE), _i32(a), _i32(b) if case["ragged"] else None
        st["out"] = torch.zeros(st["q"].shape, dtype=torch.bfloat16, device=DEVICE)
        st["max_context"] = int((a + b).max())
        if own:
            from paper_2601_17768_amd.paged import Rope
            st["cache"] = _cache(case, st["kv"], False)
            st["rope"] = Rope(case["rot"], case["theta"], max_position=int((a + b).max()) + 1, layout=case["layout"],
                              scaling=SCALINGS[case["scaling"]])
        else:
            freq, st["factor"] = _frequencies(case)
            st["freq"] = torch.tensor(freq, dtype=torch.float64, device=DEVICE)
        return st
    if case["op"] == "bounds":
        k = _bounds_inputs(case, seed)
        table, blocks = _table((a + b + BLOCK - 1) // BLOCK, seed)
        done = _touched(case)
        st["ids"] = _i32([table[s, x] for s, x in done])
        if own:
            st["cache"] = _cache(case, _paged(k, k, table, blocks), True)
            st["bt"], st["first"], st["count"] = torch.as_tensor(table, device=DEVICE), _i32(a), _i32(b)
        else:
            st["k"] = k.unflatten(2, (-1, BLOCK))
            st["seq"], st["block"] = _i32([s for s, _ in done]).long(), _i32([x for _, x in done]).long()
        return st
    k, v, st["q"], g = _context(case, seed, case["op"] == "attention")
    st["lens"], st["valid"] = _i32(a), _i32(b) if case["ragged"] else None
    st["max_context"] = int((a + b).max())
    table, blocks = _table((a + b + BLOCK - 1) // BLOCK, seed)
    if case["op"] == "select":
        st["out"] = torch.full((case["seqs"], case["window"], case["kv_heads"], case["budget"]), -1, dtype=torch.int32, device=DEVICE)
        if own:
            st["cache"], st["bt"] = _cache(case, _paged(k, k, table, blocks), True), torch.as_tensor(table, device=DEVICE)
            st["cache"].store_bounds(st["bt"], torch.zeros_like(st["lens"]), _i32(a + b), max(1, int((a + b).max())))
        else:
            lo, hi, e = _block_bounds(k[0].unflatten(1, (-1, BLOCK)))
            st["bounds"] = lo.to(torch.int8), hi.to(torch.int8), e.to(torch.int8)          # [seq][block][kv head][feature], [..][1]
        return st
    st["selected"] = _random_lists(case, g)
    st["out"] = torch.zeros_like(st["q"])
    if own:
        st["cache"], st["bt"] = _cache(case, _paged(k, v, table, blocks), False), torch.as_tensor(table, device=DEVICE)
    else:
        st["k"], st["v"] = k[0], v[0]
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------
def _frequencies(case):
    """Angle per position of every rotated pair, and the factor of the rotated values."""
    sc, rot = SCALINGS[case["scaling"]], case["rot"]
    freq = [case["theta"] ** (-2.0 * j / rot) for j in range(rot // 2)]
    if sc["kind"] == "none":
        return freq, 1.0
    f = sc["factor"]
    if sc["kind"] == "linear":
        return [x / f for x in freq], 1.0
    n = sc["original_max_position"]
    if sc["kind"] == "llama3":
        lo, hi = sc["low_freq_factor"], sc["high_freq_factor"]
        out = []
        for x in freq:
            turns = n * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - lo) / (hi - lo)))
            out.append(x * (keep + (1.0 - keep) / f))
        return out, 1.0
    at = lambda turns: rot * math.log(n / (turns * 2 * math.pi)) / (2 * math.log(case["theta"]))
    lo, hi = max(0, math.floor(at(sc["beta_fast"]))), min(rot - 1, math.ceil(at(sc["beta_slow"])))
    hi = hi + 0.001 if hi == lo else hi
    ramp = [min(1.0, max(0.0, (j - lo) / (hi - lo))) for j in range(rot // 2)]
    return [x * (1.0 - r) + x / f * r for x, r in zip(freq, ramp)], 0.1 * math.log(f) + 1.0


def _plain_rotated(x, gain, cos, sin, case):
    """x [seq, row, head, feature] in fp32: normed, then its first `rot` features rotated."""
    x = x.float()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    rot = case["rot"]
    if case["layout"] == "half":
        one, two = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((one * cos - two * sin, two * cos + one * sin), -1)
    else:
        one, two = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((one * cos - two * sin, two * cos + one * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _k_at(hd):
    t, f = torch.arange(16, device=DEVICE)[:, None], torch.arange(hd, device=DEVICE)
    return (f // 8 * 16 + t) * 8 + f % 8


def _v_at(hd):
    t, f = torch.arange(16, device=DEVICE)[:, None], torch.arange(hd, device=DEVICE)
    return ((f // 16 * 4 + t // 4) * 16 + f % 16) * 4 + t % 4


def _block_bounds(k):
    """k [..., 16, kv_heads, hd] -> lo, hi [..., kv_heads, hd] in whole multiples of 2^e, e [..., kv_heads, 1] (fp32 all)."""
    hi, lo = k.amax(-3).float(), k.amin(-3).float()
    top = torch.maximum(hi, -lo).amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                              # top = m 2^e, m in [1/2, 1)
    e = torch.where(top > 0, e - 7 + (m > 127 / 128).int(), -40).clamp_(min=-40)
    unit = torch.ldexp(torch.ones_like(top), -e)
    return torch.floor(lo * unit), torch.ceil(hi * unit), e.float()


def _plain_select(st):
    case, out = st["case"], st["out"]
    n, w, h, g, hd = case["seqs"], case["window"], case["kv_heads"], case["group"], case["hd"]
    lo, hi, e = (x.float() for x in st["bounds"])
    blocks = lo.shape[1]
    q = st["q"].float()
    top = q.abs().amax(-1, keepdim=True)
    m, qe = torch.frexp(top)
    qe = torch.where(top > 0, qe - 7 + (m > 127 / 128).int(), -40).clamp_(min=-40)
    q = torch.round(q * torch.ldexp(torch.ones_like(top), -qe))
    q = q.view(n, w, h, g, hd).permute(0, 2, 1, 3, 4).reshape(n * h, w * g, hd)
    lo, hi = (x.permute(0, 2, 3, 1).reshape(n * h, hd, blocks) for x in (lo, hi))
    dot = (q.clamp(min=0) @ hi + q.clamp(max=0) @ lo).view(n, h, w, g, blocks)
    unit = torch.exp2(qe.view(n, w, h, g, 1).permute(0, 2, 1, 3, 4) + e.permute(0, 2, 3, 1).view(n, h, 1, 1, blocks))
    score = (dot * unit).amax(3)                                                                # [seq][kv head][row][block]
    at = torch.arange(blocks, device=out.device)
    row = torch.arange(w, device=out.device)
    mine = ((st["lens"].long()[:, None] + row) // BLOCK)[:, None, :, None]
    score = score.masked_fill((at < case["sink"]) | (at > mine - case["recent"]), math.inf).masked_fill(at > mine, -math.inf)
    best, ids = score.sort(stable=True, dim=-1, descending=True)
    best, ids = best[..., :case["budget"]], ids[..., :case["budget"]]
    ids = ids.masked_fill(best == -math.inf, blocks).sort(-1).values
    ids = torch.where(ids == blocks, -1, ids).permute(0, 2, 1, 3).int()
    ids = torch.nn.functional.pad(ids, (0, case["budget"] - ids.shape[-1]), value=-1)
    if st["valid"] is not None:
        ids = torch.where((row < st["valid"][:, None])[..., None, None], ids, out)
    return out.copy_(ids)


def _plain_attention(st):
    case, out = st["case"], st["out"]
    n, w, h, g, hd = case["seqs"], case["window"], case["kv_heads"], case["group"], case["hd"]
    row = torch.arange(w, device=out.device)
    k, v = (x.unflatten(1, (-1, BLOCK)) for x in (st["k"], st["v"]))                            # [seq][block][16][kv head][feature]
    sel = st["selected"].long()
    s = torch.arange(n, device=out.device)[:, None, None, None]
    hh = torch.arange(h, device=out.device)[:, None]
    pos = st["lens"].long()[:, None] + row
    at = sel[..., None] * BLOCK + torch.arange(BLOCK, device=out.device)                        # [seq][row][kv head][entry][16]
    seen = ((sel >= 0)[..., None] & (at <= pos[:, :, None, None, None])).flatten(3)
    ids = sel.clamp(0, k.shape[1] - 1)
    kk = k.permute(0, 3, 1, 2, 4)[s, hh, ids].float().reshape(n * w * h, -1, hd)
    sc = st["q"].float().view(n * w * h, g, hd) @ kk.transpose(1, 2).contiguous() / math.sqrt(hd)
    del kk
    sc = sc.masked_fill(~seen.reshape(n * w * h, 1, -1), -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    vv = v.permute(0, 3, 1, 2, 4)[s, hh, ids].float().reshape(n * w * h, -1, hd)
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, p @ vv / total, 0.0).view(out.shape).to(out.dtype)
    if st["valid"] is not None:
        o = torch.where((row < st["valid"][:, None])[..., None, None], o, out)
    return out.copy_(o)


def _plain_append(st):
    case, out, kv = st["case"], st["out"], st["kv"]
    row = torch.arange(case["window"], device=out.device)
    pos = st["lens"].long()[:, None] + row
    angle = (pos.double()[..., None] * st["freq"])[:, :, None]
    cos, sin = (torch.cos(angle) * st["factor"]).float(), (torch.sin(angle) * st["factor"]).float()
    there = torch.ones_like(pos, dtype=torch.bool) if st["valid"] is None else row < st["valid"][:, None]
    out.copy_(torch.where(there[..., None, None], _plain_rotated(st["q"], st["norms"][0], cos, sin, case).to(out.dtype), out))
    k = _plain_rotated(st["k"], st["norms"][1], cos, sin, case).to(kv.dtype)
    block = torch.gather(st["bt"].long(), 1, (pos // BLOCK).clamp(max=st["bt"].shape[1] - 1))
    s, i = torch.nonzero(there, as_tuple=True)
    head = torch.arange(case["kv_heads"], device=out.device)[:, None]
    b, t = block[s, i][:, None, None], pos[s, i] % BLOCK
    kv[0, 0].index_put_((b, head, _k_at(case["hd"])[t][:, None]), k[s, i])
    kv[0, 1].index_put_((b, head, _v_at(case["hd"])[t][:, None]), st["v"][s, i].to(kv.dtype))
    return out, kv


def _bound_values(lo, hi, e):
    unit = torch.exp2(e)
    return (lo * unit).to(torch.bfloat16), (hi * unit).to(torch.bfloat16)


def run(state):
    case = state["case"]
    if case["op"] == "append":
        if not own:
            return _plain_append(state)
        cache = state["cache"]
        cache.append(0, state["k"], state["v"], state["bt"], state["lens"], q=state["q"], q_out=state["out"], n_valid=state["valid"],
                     max_context=state["max_context"], rope=state["rope"], q_norm=state["norms"][0], k_norm=state["norms"][1], eps=EPS)
        return state["out"], cache.kv
    if case["op"] == "bounds":
        if own:
            state["cache"].store_bounds(state["bt"], state["first"], state["count"], case["hi"])
            return state["cache"].read_bounds(state["ids"])
        return _bound_values(*_block_bounds(state["k"][:, state["seq"], state["block"]]))
    if case["op"] == "select":
        if own:
            return state["cache"].select(0, state["q"], state["bt"], state["lens"], case["budget"], sink=case["sink"], recent=case["recent"],
                                         n_valid=state["valid"], max_context=state["max_context"], selected=state["out"])
        return _plain_select(state)
    if own:
        return state["cache"].attention(0, state["q"], state["bt"], state["lens"], state["selected"], n_valid=state["valid"],
                                        max_context=state["max_context"], out=state["out"])
    return _plain_attention(state)


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _defined_bounds(k):
    """k [16, ..., hd] float64 -> smallest and largest of every feature, outward to whole multiples of the block's power of two."""
    top = k.abs().amax(0).amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 127.0)).clamp(min=-40.0)
    e = torch.where(top <= 127.0 * torch.exp2(e - 1), e - 1, e).clamp(min=-40.0)          # (the logarithm of a border is not)
    e = torch.where(top > 127.0 * torch.exp2(e), e + 1, e)
    unit = torch.exp2(e)
    return torch.floor(k.amin(0) / unit) * unit, torch.ceil(k.amax(0) / unit) * unit


def _defined_turned(x, gain, pos, case):
    """x [row, head, hd] float64 at positions pos, as complex numbers."""
    if gain is not None:
        x = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * gain.double()
    rot = case["rot"]
    freq, factor = _frequencies(case)
    turn = torch.polar(torch.full((len(pos), rot // 2), factor, dtype=torch.float64, device=DEVICE),
                       torch.outer(pos.double(), torch.tensor(freq, dtype=torch.float64, device=DEVICE)))[:, None]
    x = x.clone()
    if case["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
        x[..., :rot] = torch.view_as_real(z).flatten(-2)
    return x


def _exact_append(case, seed):
    q, k, v, norms, kv, table = _append_inputs(case, seed)
    a, b = _lengths(case)
    out, kv = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE), kv.double()
    hd = case["hd"]
    for s in range(case["seqs"]):
        f, n = int(a[s]), int(b[s])
        if not n:
            continue
        pos = torch.arange(f, f + n, device=DEVICE)
        out[s, :n] = _defined_turned(q[s, :n].double(), norms[0], pos, case)
        kk, vv = _defined_turned(k[s, :n].double(), norms[1], pos, case), v[s, :n].double()
        for x in range(f // BLOCK, (f + n - 1) // BLOCK + 1):
            p0, p1 = max(f, x * BLOCK), min(f + n, (x + 1) * BLOCK)
            for plane, new in ((0, kk), (1, vv)):
                tile = kv[0, plane, int(table[s, x])]
                t = tile.view(-1, hd // 8, 16, 8).transpose(1, 2) if plane == 0 else tile.view(-1, hd // 16, 4, 16, 4).permute(0, 2, 4, 1, 3)
                t = t.reshape(-1, 16, hd).clone()                                          # [kv head][token][feature]
                t[:, p0 - x * BLOCK:p1 - x * BLOCK] = new[p0 - f:p1 - f].transpose(0, 1)
                if plane == 0:
                    tile.copy_(t.view(-1, 16, hd // 8, 8).transpose(1, 2).reshape(tile.shape))
                else:
                    tile.copy_(t.view(-1, 4, 4, hd // 16, 16).permute(0, 3, 1, 4, 2).reshape(tile.shape))
    return out, kv


def exact(case, seed):
    a, b = _lengths(case)
    if case["op"] == "append":
        return _exact_append(case, seed)
    if case["op"] == "bounds":
        k = _bounds_inputs(case, seed)
        done = _touched(case)
        lo = torch.zeros((case["layers"], len(done), case["kv_heads"], case["hd"]), dtype=torch.float64, device=DEVICE)
        hi = torch.zeros_like(lo)
        for i in range(case["layers"] if done else 0):
            lo[i], hi[i] = _defined_bounds(torch.stack([k[i, s, x * BLOCK:(x + 1) * BLOCK] for s, x in done], 1).double())
        return lo, hi
    k, v, q, g = _context(case, seed, case["op"] == "attention")
    n, w, h, group, hd = case["seqs"], case["window"], case["kv_heads"], case["group"], case["hd"]
    if case["op"] == "select":
        out = torch.full((n, w, h, case["budget"]), -1, dtype=torch.int32, device=DEVICE)
        for s in range(n):
            if not b[s]:
                continue
            lo, hi = _defined_bounds(k[0, s].double().unflatten(0, (-1, BLOCK)).transpose(0, 1))     # [block][kv head][feature]
            for i in range(int(b[s])):
                mine = (int(a[s]) + i) // BLOCK
                x = q[s, i].double()
                top = x.abs().amax(-1, keepdim=True)
                unit = torch.exp2(torch.ceil(torch.log2(top / 127.0)).clamp(min=-40.0))
                unit = torch.where((top <= 63.5 * unit) & (unit > 2.0 ** -40), unit / 2, torch.where(top > 127.0 * unit, unit * 2, unit))
                x = (torch.round(x / unit) * unit).view(h, group, 1, hd)
                lo_, hi_ = lo[:mine + 1].transpose(0, 1)[:, None], hi[:mine + 1].transpose(0, 1)[:, None]    # [kv head][1][block][feature]
                score = torch.cat([torch.maximum(x * lo_[:, :, c:c + 4096], x * hi_[:, :, c:c + 4096]).sum(-1).amax(1)
                                   for c in range(0, mine + 1, 4096)], -1).cpu().numpy()
                for j in range(h):
                    forced = [y for y in range(mine + 1) if y < case["sink"] or y > mine - case["recent"]][:case["budget"]]
                    others = np.setdiff1d(np.arange(mine + 1), forced)
                    best = others[np.argsort(-score[j, others], kind="stable")][:max(0, min(case["budget"], mine + 1) - len(forced))]
                    ids = np.sort(np.concatenate([np.asarray(forced, np.int64), best]))
                    out[s, i, j, :len(ids)] = torch.as_tensor(ids.astype(np.int32), device=DEVICE)
        return out
    sel = _random_lists(case, g)
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    step = torch.arange(BLOCK, device=DEVICE)
    for s in range(n):
        kd, vd = (x[0, s].double().transpose(0, 1) for x in (k, v))                                  # [kv head][token][feature]
        for i in range(int(b[s])):
            last = int(a[s]) + i
            ids = sel[s, i].long()
            at = torch.where(ids < 0, last + 1, ids * BLOCK)[..., None] + step
            at = at.flatten(1)                                                                      # [kv head][key]
            hidden = at > last
            at = at.clamp(max=kd.shape[1] - 1)[..., None].expand(-1, -1, hd)
            z = q[s, i].double().view(h, group, hd) @ torch.gather(kd, 1, at).transpose(1, 2) * hd ** -0.5
            out[s, i] = (torch.softmax(z.masked_fill(hidden[:, None], -math.inf), -1) @ torch.gather(vd, 1, at)).view(h * group, hd)
    return out
