"""The decoding step with attention over selected blocks: calls whose result may depend on nothing but their inputs."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from helpers import wl
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd import kv_layout
from paper_2601_17768_amd.paged import PagedCache
from paper_2601_17768_amd.session import VerifierSession
from test_gpu_kv4_step import VOCAB, cached_kv, factor, mirror_model
from test_gpu_sparse_step import EPS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


@pytest.mark.parametrize("hd,kv_heads,group,longest", [(128, 2, 4, 2000), (64, 2, 2, 6000)])
def test_blocks_with_infinite_bounds_and_a_workspace_that_holds_anything(hd, kv_heads, group, longest):
    """Every block's bounds say -infinity .. infinity: the lowest blocks are read, whatever the workspace held.  (Rows picked by waves; the bounds are
    written by hand, so that the attention itself stays one of ordinary numbers.)  Tolerance: as in test_gpu_sparse_step."""
    shape, w = mirror_model(kv_heads, group, hd)
    max_context = longest + 16
    sess = VerifierSession(shape, w, max_position=max_context, device=DEV)
    g, rng = torch.Generator().manual_seed(hd), wl.rng_for(hd, 4)
    lens = [longest - 1, longest // 2, 700]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=2, max_blocks_per_seq=-(-max_context // 16))
    bt, kv, cached = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks), []
    for s, n in enumerate(lens):
        k, v = cached_kv(shape, n, g)
        cached.append((k, v))
        kv_layout.write_tokens(kv, bt[s], *(torch.cat((t[None], torch.zeros(group, *t.shape, dtype=t.dtype))) for t in (k, v)))
    cache, seq, tok = sess.paged(kv), i32(lens), i32(rng.integers(0, VOCAB, len(lens)))
    rec = cache.bounds.view(-1, 2 * hd + 16)
    rec.zero_()
    rec[:, 2 * hd] = 255
    budget, sink, recent = 9, 2, 1
    start, seen = kv.clone(), []
    for fill in (0, 1, 255, 3):
        sess.decode_sparse(cache, bt, seq, tok, budget, sink, recent, max_context=max_context)
        kv.copy_(start)
        rec.zero_()
        rec[:, 2 * hd] = 255
        sess._ws.fill_(fill)
        out = sess.decode_sparse(cache, bt, seq, tok, budget, sink, recent, max_context=max_context)
        seen.append((out.clone(), kv.clone()))
    for out, after in seen[1:]:
        assert torch.equal(out, seen[0][0]) and torch.equal(after, seen[0][1])
    for s, n in enumerate(lens):
        k, v = (x[:, n].cpu() for x in kv_layout.read_tokens(seen[0][1], bt[s], n + 1, hd))
        keys, values = torch.cat((cached[s][0], k[:1])), torch.cat((cached[s][1], v[:1]))
        listed = list(range(budget - recent)) + [n // 16]
        outs, mags = [], []
        for h in range(kv_heads):
            q = torch.stack([(keys[-1, h].double() * factor(h * group + j, group)).to(torch.bfloat16) for j in range(group)])
            a, mag = ref.attention(q, keys[:, h], values[:, h], listed, n, hd ** -0.5)
            outs.append(a)
            mags.append(mag)
        a, mag = torch.cat(outs).flatten(), torch.cat(mags).flatten()
        t = 2.0 ** -8 * a.abs() + 2.0 ** -12 * mag
        x = w["embed"][int(tok[s])].double() + a
        rms, r = torch.sqrt((x * x).mean() + EPS), t.norm() / x.norm()
        want = x / rms
        tol = (t + x.abs() * r) / (rms * (1 - r)) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 1e-6
        assert bool(((v[1:].flatten().double() - want).abs() <= tol).all()), (s, n)
    sess.close()


def test_heads_that_are_not_the_models_are_refused():
    """A cache of the same bytes in another layout: a kv head of 128 features for two of 64, whose records of bounds take less room; and of other query heads."""
    shape = wl.TINY.replace(n_q_heads=4, n_kv_heads=2, head_dim=64)
    sess = VerifierSession(shape, wl.make_weights(shape, seed=3), max_position=128, device=DEV)
    assert bytes(B.llm42_model_heads(sess.model)) == bytes(B.Heads(shape.n_layers, 4, 2, 64))
    kv = sess.kv_cache(4)
    other = kv.view(shape.n_layers, 2, 4, 1, 16 * 128)
    bt, zero = i32([[0, 1, 2, 3]]), i32([0])
    for cache in (PagedCache(other, 2, 128), PagedCache(kv, 8, 64), PagedCache(kv[:1], 4, 64)):
        before = cache.bounds.fill_(3).clone()
        with pytest.raises(ValueError):
            sess.decode_sparse(cache, bt, zero, zero, 2, 0, 1)
        assert torch.equal(cache.bounds, before)
    sess.decode_sparse(sess.paged(kv), bt, zero, zero, 2, 0, 1)
    sess.close()


def test_one_workspace_serves_fewer_sequences_and_shorter_contexts():
    """Across the context lengths at which attention over the whole context would change the way in which it is split (8 kv heads, one sequence: 47104)."""
    shape = wl.TINY.replace(d_model=512, n_q_heads=8, n_kv_heads=8, head_dim=128)
    sess = VerifierSession(shape, wl.make_weights(shape, seed=4), max_position=60000, device=DEV)
    contexts = [1, 16, 17, 255, 257, 2048, 2049, 8000, 8192, 8208, 16000, 40960, 45056, 47104, 47105, 49152, 59999, 60000]
    need = lambda n, c, b: B.llm42_decode_step_sparse_workspace_bytes(sess.model, n, c, b)
    for budget in (4, 64, 2000):
        for n in (1, 2, 5, 24, 130):
            sizes = [need(n, c, budget) for c in contexts]
            assert sizes == sorted(sizes)
            assert sizes[-1] <= need(n + 1, contexts[-1], budget)
    bt, one = i32(np.arange(3750)[None]), i32([40])
    kv = sess.kv_cache(3750)
    kv.normal_(generator=torch.Generator(device=DEV).manual_seed(2))
    cache = sess.paged(kv)
    cache.store_bounds(bt, i32([0]), one, 40)
    ws, out, seen = torch.empty(need(1, 49152, 64), dtype=torch.uint8, device=DEV), i32([-7]), []
    for c in (49152, 47104, 41):
        start = kv.clone()
        B.llm42_decode_step_sparse(sess.model, cache.heads, kv, 3750, bt, cache.bounds, 64, 1, 2, one, i32([5]), c, out, ws)
        seen.append((int(out), kv.clone()))
        kv.copy_(start)
    assert all(t == seen[0][0] and torch.equal(after, seen[0][1]) for t, after in seen)
    sess.close()


def test_the_workspace_holds_no_partials_of_the_whole_context():
    """128 sequences of 131072 positions: the scores of 8192 blocks for each kv head, the lists, and what a step takes at a context of one block."""
    shape = wl.TINY.replace(d_model=512, n_q_heads=8, n_kv_heads=8, head_dim=128)
    sess = VerifierSession(shape, wl.make_weights(shape, seed=4), max_position=131072, device=DEV)
    need = lambda c: B.llm42_decode_step_sparse_workspace_bytes(sess.model, 128, c, 64)
    assert need(131072) - need(16) <= 4 * 128 * 8 * 8192 + 4096
    sess.close()


def test_sequences_that_are_not_in_order_store_no_bounds():
    """Whose token would have made a block whole: each with one thing wrong, in a block before that one."""
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=512, device=DEV)
    rng = wl.rng_for(6, 2)
    lens = [303, 303, 47, 47, 47]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    cache, seq = sess.paged(kv), i32(lens)
    cache.bounds.fill_(77)
    cache.store_bounds(bt, torch.zeros_like(seq), seq, 303)
    before, start = cache.bounds.clone().view(shape.n_layers, blocks, -1), kv.clone()
    whole = [int(table[s][lens[s] // 16]) for s in range(5)]
    assert bool((before[:, whole] == 77).all())
    bad_bt, bad_tok = bt.clone(), tok.clone()
    bad_bt[1, 3], bad_bt[2, 0] = blocks, -1
    bad_tok[3] = -1
    status = i32([9] * 5)
    out = sess.decode_sparse(cache, bad_bt, seq, bad_tok, 4, seq_status=status)
    assert status.tolist() == [0, B.LLM42_SEQ_BAD_BLOCK, B.LLM42_SEQ_BAD_BLOCK, B.LLM42_SEQ_BAD_TOKEN, 0] and out[1:4].tolist() == [-1] * 3
    after = cache.bounds.view(shape.n_layers, blocks, -1)
    moved = (after != before).any(-1)
    assert bool(moved[:, [whole[0], whole[4]]].all()) and int(moved.sum()) == 2 * shape.n_layers
    changed = (kv != start).any(-1).any(-1).any(0).any(0).nonzero().flatten().tolist()
    assert sorted(changed) == sorted([whole[0], whole[4]])
    sess.close()
