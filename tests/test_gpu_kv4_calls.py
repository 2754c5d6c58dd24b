"""Calls of the 4-bit cache that reach past one launch, share blocks, or change stream."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
from helpers import wl
from paper_2601_17768_amd import dvr, kv_layout
from paper_2601_17768_amd.session import VerifierSession

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


def session(kv_heads, group, hd, layers):
    shape = wl.ModelShape(n_layers=layers, d_model=128, n_q_heads=kv_heads * group, n_kv_heads=kv_heads, head_dim=hd, d_ffn=64, vocab=16,
                          rope_theta=1e4)
    return VerifierSession(shape, wl.make_weights(shape), max_position=1024, device=DEV)


@pytest.mark.parametrize("hd", [64, 128])
def test_store_and_read_of_more_workgroups_than_a_launch_takes(hd):
    """2^24 + 5 sequences (a launch takes 2^24 - 1 workgroups of 256): most of them empty, some at both ends and on the border stored."""
    sess, num = session(1, 1, hd, 1), 2 ** 24 + 5
    at = [0, 1, 2 ** 24 - 2, 2 ** 24 - 1, 2 ** 24, num - 1]
    g = torch.Generator().manual_seed(hd)
    k, v = (torch.randn(1, 16 * len(at), 1, hd, generator=g).to(torch.bfloat16) for _ in range(2))
    kv, blocks = sess.kv_cache(len(at)), torch.arange(len(at), device=DEV)
    kv_layout.write_tokens(kv, blocks, k, v)
    bt, first, count = i32([0]).repeat(num, 1), i32([3]).repeat(num), i32([0]).repeat(num)
    bt[at, 0], count[at] = blocks.int(), 1
    first[at] = i32([5, 0, 15, 7, 8, 2])
    kv4, status = sess.kv4_cache(len(at)), i32([9]).repeat(num)
    kv4.fill_(255)
    sess.kv4_store(kv, kv4, bt, first, count, 1, seq_status=status)
    assert not bool(status.any())
    status.fill_(9)
    ok, ov = (torch.full((1, num, 1, 1, hd), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    sess.kv4_read(kv4, bt, first, count, 1, ok, ov, seq_status=status)
    assert not bool(status.any())
    rows = torch.arange(len(at)) * 16 + first[at].cpu()
    for got, x in ((ok, k), (ov, v)):
        assert torch.equal(got[0, at, 0, 0].cpu(), ref.quantized(x[0, rows, 0]).to(torch.bfloat16))
        got[:, at] = 5.0
        assert bool((got == 5.0).all())
    sess.close()


def test_calls_of_a_session_on_two_streams_follow_each_other():
    """They share its workspace.  A stream that is held back is used first, then another one: the second call ends behind the first, and a
    workspace that the held-back stream still uses is not handed out when it is outgrown."""
    sess = session(2, 4, 128, 1)
    g = torch.Generator().manual_seed(1)
    kv = torch.randn(tuple(sess.kv_cache(300).shape), generator=g).to(torch.bfloat16).to(DEV)
    kv4, bt = sess.kv4_cache(300), torch.arange(300, dtype=torch.int32, device=DEV).view(1, 300)
    sess.kv4_store(kv, kv4, bt, i32([0]), i32([4800]), 4800)
    q = [torch.randn(1, w, 8, 128, generator=g).to(torch.bfloat16).to(DEV) for w in (1, 1, 40)]
    lens, out = i32([4700]), [torch.zeros_like(x) for x in q]
    want = [sess.kv4_attention(0, kv4, bt, x, lens) for x in q]
    sess._ws, side = None, torch.cuda.Stream()
    sess.kv4_attention(0, kv4, bt, q[0], lens, out=out[0])       # (in parts: the workspace is written)
    first = sess._ws.data_ptr(), sess._ws.numel()
    assert first[1] > 8 * 128 * 4 * 4
    torch.cuda.synchronize()
    ends = [torch.cuda.Event(), torch.cuda.Event()]
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        sess.kv4_attention(0, kv4, bt, q[0], lens, out=out[0])
        ends[0].record()
    sess.kv4_attention(0, kv4, bt, q[1], lens, out=out[1])
    ends[1].record()
    ends[1].synchronize()
    assert ends[0].query()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        sess.kv4_attention(0, kv4, bt, q[0], lens, out=out[0])
        ends[0].record()
        sess.kv4_attention(0, kv4, bt, q[2], lens, out=out[2])   # outgrows the workspace, which the default stream allocated
    taken = [torch.empty(first[1], dtype=torch.uint8, device=DEV) for _ in range(4)]
    pending = not ends[0].query()
    assert sess._ws.data_ptr() != first[0] and pending and all(t.data_ptr() != first[0] for t in taken)
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
    sess.close()


def test_a_shared_prefix_is_stored_from_every_sequence_and_the_loop_runs_on_it():
    """Three sequences whose tables begin with the same three blocks: the cache holds what one of them stores alone, and the loop releases the
    verifier's stream."""
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=42), max_position=512, device=DEV)
    rng = wl.rng_for(7, 1)
    common, tails = wl.random_tokens(rng, 48, shape.vocab), [wl.random_tokens(rng, n, shape.vocab) for n in (5, 22, 16)]
    bt = torch.arange(36, dtype=torch.int32, device=DEV).view(3, 12)
    bt[1:, :3] = bt[0, :3]

    def state():
        kv = sess.kv_cache(36)
        sess.prefill(kv, bt[:1].contiguous(), [common], window=16)
        first = sess.prefill(kv, bt, tails, window=16, cached=i32([48] * 3))
        return kv, bt, i32([48 + len(t) for t in tails]), first

    kv, _, lens, first = state()
    kv4, alone = sess.kv4_cache(36), sess.kv4_cache(36)
    for cache in (kv4, alone):
        cache.fill_(255)
    sess.kv4_store(kv, kv4, bt, i32([0] * 3), lens, 80)
    sess.kv4_store(kv, alone, bt[:1].contiguous(), i32([0]), lens[:1].contiguous(), 80)
    sess.kv4_store(kv, alone, bt, i32([48] * 3), lens - 48, 80)
    assert torch.equal(kv4, alone)
    want = dvr.generate_verifier_only(sess, *state(), 24)
    got, _ = dvr.generate(sess, *state(), 24, 8, fast="mx4_cache")
    assert torch.equal(got, want)
    sess.close()
