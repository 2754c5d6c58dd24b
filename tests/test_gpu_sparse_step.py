"""The decoding step with attention over selected blocks: its attention by value, for selections made in LDS and through the workspace, whole lists and lists in
parts; the bounds that it keeps up; sequences that are not in order; the decode - verify - rollback loop on it.

The attention is made visible by the model of test_gpu_kv4_step: the bf16 cache shows the query and (embedding + attention) / rms."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from helpers import wl
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd import dvr, kv_layout
from paper_2601_17768_amd.session import VerifierSession
from test_gpu_kv4_step import EPS, VOCAB, cached_kv, factor, mirror_model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


def expected(shape, e, k, v, budget, sink, recent):
    """What the later layers' values show, and how far it may be off.  k, v [keys, kv heads, hd], the newest last.  The weights of the attention enter in two bf16
    parts and its sums are fp32 (2^-12 of the weighted magnitudes), its output is rounded to bf16; from there on as a residual's error spreads: its norm
    shifts the rms by |t| / |x| of it at most; the normed row is rounded to bf16."""
    group, pos = shape.n_q_heads // shape.n_kv_heads, len(k) - 1
    outs, mags = [], []
    for h in range(shape.n_kv_heads):
        q = torch.stack([(k[-1, h].double() * factor(h * group + j, group)).to(torch.bfloat16) for j in range(group)])
        bounds = [ref.bounds(k[16 * b:16 * b + 16, h]) for b in range(pos // 16 + 1)]
        lo, hi = (torch.stack([x[i] for x in bounds]) for i in range(2))
        blocks = ref.select(q, lo, hi, pos // 16, budget, sink, recent)
        a, mag = ref.attention(q, k[:, h], v[:, h], blocks, pos, shape.head_dim ** -0.5)
        outs.append(a)
        mags.append(mag)
    a, mag = torch.cat(outs).flatten(), torch.cat(mags).flatten()
    t = 2.0 ** -8 * a.abs() + 2.0 ** -12 * mag
    x = e.double() + a
    rms, r = torch.sqrt((x * x).mean() + EPS), t.norm() / x.norm()
    want = x / rms
    return want, (t + x.abs() * r) / (rms * (1 - r)) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 1e-6


# (hd, kv heads, group, sequences, max_context, longest, budget, sink, recent): on 256 CUs
CASES = [
    (128, 2, 4, 5, 3008, 3000, 16, 1, 2), (64, 2, 4, 24, 3008, 900, 8, 0, 1), (128, 1, 8, 3, 6000, 5990, 100, 4, 8), (64, 2, 3, 6, 4096, 4090, 128, 1, 2),
    (64, 2, 5, 2, 65536, 20000, 40, 1, 2), (128, 2, 2, 3, 40000, 10000, 300, 0, 30), (128, 2, 1, 260, 1024, 400, 5, 1, 1), (64, 2, 4, 40, 512, 500, 64, 1, 2),
]


@pytest.mark.parametrize("hd,kv_heads,group,num,max_context,longest,budget,sink,recent", CASES)
def test_attention_of_the_sparse_step(hd, kv_heads, group, num, max_context, longest, budget, sink, recent):
    shape, w = mirror_model(kv_heads, group, hd)
    sess = VerifierSession(shape, w, max_position=max_context, device=DEV)
    g, rng = torch.Generator().manual_seed(num + hd), wl.rng_for(num, hd)
    lens = [longest, longest // 16 * 16 - 1, 0, 15, 16, 31, longest // 2][:num]
    lens += [int(x) for x in rng.integers(0, min(longest, 700), num - len(lens))]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=2, max_blocks_per_seq=-(-max_context // 16))
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    cached = []
    for s, n in enumerate(lens):
        k, v = cached_kv(shape, n, g)
        cached.append((k, v))
        if n:
            kv_layout.write_tokens(kv, bt[s], *(torch.cat((t[None], torch.zeros(group, *t.shape, dtype=t.dtype))) for t in (k, v)))
    cache, seq, tok = sess.paged(kv), i32(lens), i32(rng.integers(0, VOCAB, num))
    cache.bounds.fill_(77)
    cache.store_bounds(bt, torch.zeros_like(seq), seq, max(lens))
    before, status = cache.bounds.clone(), i32([9] * num)
    out = sess.decode_sparse(cache, bt, seq, tok, budget, sink, recent, max_context=max_context, seq_status=status).clone()
    assert not bool(status.any())
    for s, n in enumerate(lens):
        k, v = (x[:, n].cpu() for x in kv_layout.read_tokens(kv, bt[s], n + 1, hd))
        want, tol = expected(shape, w["embed"][int(tok[s])], torch.cat((cached[s][0], k[:1])), torch.cat((cached[s][1], v[:1])), budget, sink, recent)
        err = (v[1:].flatten().double() - want).abs()
        assert bool((err <= tol).all()), (s, n, float((err / tol).max()))
    # the bounds of the blocks that became whole, in every layer, and no others
    after = cache.bounds.clone()
    cache.bounds.copy_(before)
    cache.store_bounds(bt, seq, torch.ones_like(seq), 1)
    assert torch.equal(cache.bounds, after)
    # the same call gives the same bits, eager and replayed
    held = kv.clone()
    again = torch.empty_like(out)
    step = lambda: sess.decode_sparse(cache, bt, seq, tok, budget, sink, recent, max_context=max_context, out_tokens=again)
    step()
    assert torch.equal(again, out) and torch.equal(kv, held) and torch.equal(cache.bounds, after)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        again.fill_(-5)
        cache.bounds.copy_(before)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, out) and torch.equal(kv, held) and torch.equal(cache.bounds, after)
    sess.close()


def test_sequences_that_are_not_in_order_take_no_part():
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=512, device=DEV)
    rng = wl.rng_for(6, 1)
    lens = [200, 300, 63, 40, 111]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    cache, seq = sess.paged(kv), i32(lens)
    cache.store_bounds(bt, torch.zeros_like(seq), seq, 300)
    start, bounds = kv.clone(), cache.bounds.clone()
    want = sess.decode_sparse(cache, bt, seq, tok, 4).clone()
    kv.copy_(start)
    cache.bounds.copy_(bounds)
    bad_bt, bad_seq, bad_tok = bt.clone(), seq.clone(), tok.clone()
    bad_bt[1, 3], bad_seq[2], bad_tok[3] = blocks, -1, shape.vocab
    status = i32([9] * 5)
    got = sess.decode_sparse(cache, bad_bt, bad_seq, bad_tok, 4, seq_status=status)
    assert status.tolist() == [0, B.LLM42_SEQ_BAD_BLOCK, B.LLM42_SEQ_BAD_LENGTH, B.LLM42_SEQ_BAD_TOKEN, 0]
    assert got.tolist() == [int(want[0]), -1, -1, -1, int(want[4])]
    moved = (kv != start).any(-1).any(-1).any(0).any(0).nonzero().flatten().tolist()
    assert sorted(moved) == sorted(int(table[s][lens[s] // 16]) for s in (0, 4))
    assert int((cache.bounds != bounds).view(shape.n_layers, blocks, -1).any(-1).any(0).sum()) == 1       # (111 + 1 is whole)
    for kw, code in ((dict(budget=0), -1), (dict(budget=4097), -1), (dict(budget=4, sink=3, recent=2), -1), (dict(budget=4, recent=0), -1),
                     (dict(budget=4, sink=-1), -1), (dict(budget=4, max_context=513), -4)):
        with pytest.raises(B.Llm42Error) as e:
            sess.decode_sparse(cache, bt, seq, tok, **kw)
        assert e.value.status == code
    with pytest.raises(ValueError):
        sess.decode_sparse(sess.paged(kv, bounds=False), bt, seq, tok, 4)
    sess.close()


@pytest.mark.parametrize("budget,temperature", [(1, 0.0), (3, 0.0), (3, 0.8), (64, 0.0)])
def test_the_loop_on_selected_blocks_releases_the_verifiers_stream(budget, temperature):
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=9), max_position=1024, device=DEV)
    rng = wl.rng_for(9, 2)
    prompts = [wl.random_tokens(rng, int(n), shape.vocab) for n in (300, 17, 150, 64)]
    sampling = B.make_sampling(temperature, 5, torch.arange(4, device=DEV)) if temperature else None

    def state():
        lens = np.array([len(p) for p in prompts], dtype=np.int32)
        table, blocks = wl.make_block_table(wl.rng_for(9, 3), lens + 40 + 3 * 8, 16, spare_blocks=2)
        kv, bt = sess.kv_cache(blocks), torch.as_tensor(table, device=DEV)
        return kv, bt, torch.as_tensor(lens, device=DEV), sess.prefill(kv, bt, prompts, window=32, sampling=sampling)

    want = dvr.generate_verifier_only(sess, *state(), 40, sampling=sampling)
    got, stats = dvr.generate(sess, *state(), 40, 8, sampling=sampling, fast="sparse", budget=budget)
    assert torch.equal(got, want) and stats.committed + stats.rolled_back == stats.verified_rows
    if budget == 64:                                              # (every block: little is rolled back)
        assert stats.rolled_back < stats.fast_tokens / 2
    sess.close()
