"""The decoding step's attention over the 4-bit cache by value, in every way that it is split: contexts in parts and whole, workgroups of four and
of eight waves, loads past the caches.

The model makes it visible.  Embeddings are +-1, so that a normed row is its embedding and every sum of the projections is exact; the
heads of a group ask with the kv head's own key times powers of two, so that the bf16 cache shows the query; the first layer's output
projection is the identity and its MLP zero, and each later layer's value projection copies a part of the normed residual into
the bf16 cache: (embedding + attention) / rms."""
import math

import numpy as np
import pytest
import torch

import mx4_reference as ref
from helpers import wl
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd import kv_layout
from paper_2601_17768_amd.session import VerifierSession

DEV = "cuda:0"
VOCAB, EPS = 16, 1e-5
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)
BORDERS = [0, 1, 14, 15, 16, 17, 31, 47, 48, 62, 63, 64, 65, 79, 127, 128, 129, 200, 255, 256, 257, 319, 320, 447, 511, 512, 513, 575, 576, 639]


def factor(head, group):
    """What a query is its kv head's key times."""
    return 2.0 ** (head % group % 4 - 1)


def key_size(hd):
    """Of the model's keys: large enough that the newest position counts among thousands (its scores are factor * size^2 sqrt(hd))."""
    return 0.5 if hd == 128 else 0.8


def mirror_model(kv_heads, group, hd):
    width, d = kv_heads * hd, kv_heads * group * hd
    shape = wl.ModelShape(n_layers=1 + group, d_model=d, n_q_heads=kv_heads * group, n_kv_heads=kv_heads, head_dim=hd, d_ffn=64, vocab=VOCAB,
                          rope_theta=1e4, rms_eps=EPS)
    g = torch.Generator().manual_seed(kv_heads * 1000 + group * 10 + hd)
    bf = lambda t: t.to(torch.bfloat16).contiguous()
    zeros, ones = lambda *s: torch.zeros(*s, dtype=torch.bfloat16), torch.ones(d, dtype=torch.bfloat16)
    wk, wv = (bf(torch.randn(width, d, generator=g) * (s / math.sqrt(d))) for s in (key_size(hd), 1.0))
    layers = []
    for l in range(1 + group):
        wq = torch.cat([wk[h // group * hd:(h // group + 1) * hd] * factor(h, group) for h in range(kv_heads * group)])
        pick = zeros(width, d)
        pick[torch.arange(width), (l - 1) * width + torch.arange(width)] = 1.0
        layers.append({"attn_norm": ones, "ffn_norm": ones, "wq": bf(wq) if l == 0 else zeros(d, d), "wk": wk if l == 0 else zeros(width, d),
                       "wv": wv if l == 0 else pick, "wo": bf(torch.eye(d)) if l == 0 else zeros(d, d), "w_gate": zeros(64, d), "w_up": zeros(64, d),
                       "w_down": zeros(d, 64)})
    embed = bf(torch.randint(0, 2, (VOCAB, d), generator=g) * 2.0 - 1.0)
    return shape, {"embed": embed, "final_norm": ones, "lm_head": bf(torch.randn(VOCAB, d, generator=g)), "layers": layers}


def cached_kv(shape, n, g):
    k = torch.randn(n, shape.n_kv_heads, shape.head_dim, generator=g) * 1.5
    v = torch.randn(n, shape.n_kv_heads, shape.head_dim, generator=g) * torch.exp2(torch.randint(-2, 3, (n, 1, 1), generator=g).float())
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def normed(shape, e, k, v, keep=None):
    """What the later layers' values show, and how far it may be off.  e: the embedding; k, v [keys, kv heads, hd], the newest last; keep: keys
    that count (a mistake to be found).  Attention: a weight is rounded to bf16 (2^-8 of it), the output too, exp2 and sums far below;
    a residual's error of t in each element shifts its rms by |t| / |x| of it at most; the normed row is rounded to bf16."""
    group = shape.n_q_heads // shape.n_kv_heads
    q = torch.stack([k[-1, h // group].double() * factor(h, group) for h in range(shape.n_q_heads)])
    kq, vq = ref.quantized(k), ref.quantized(v)
    if keep is not None:
        kq, vq = kq[keep], vq[keep]
    a, mag = ref.attention(q[None], kq, vq, kq.shape[0])
    a, t = a.flatten(), (2.0 ** -8 * mag + 2.0 ** -8 * a.abs() + 2.0 ** -14 * mag).flatten()
    x = e.double() + a
    rms, r = torch.sqrt((x * x).mean() + EPS), t.norm() / x.norm()
    want = x / rms
    return want, (t + x.abs() * r) / (rms * (1 - r)) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 1e-6


@pytest.mark.parametrize("hd,group", [(64, 4), (128, 4), (64, 3), (128, 8)])
def test_a_key_that_is_left_out_shows(hd, group):
    """Mistakes planted in the reference, without a GPU: without the newest position, without a part, without the first step of keys (of
    few enough keys that 64 weigh something)."""
    shape, w = mirror_model(2, group, hd)
    g = torch.Generator().manual_seed(3)
    for n in (40, 128, 700, 3000):
        k, v = cached_kv(shape, n + 1, g)
        k[-1] = (k[-1] / 1.5 * key_size(hd)).to(torch.bfloat16)   # (the size of the model's own)
        want, tol = normed(shape, w["embed"][5], k, v)
        at = torch.arange(n + 1)
        for keep in (at < n, at >= 64, (at < n // 64 * 64 // 2) | (at >= n // 64 * 64 // 2 + 512)):
            if bool(keep.any()) and not bool(keep.all()) and (n <= 700 or int(keep.sum()) != n - 63):
                wrong, _ = normed(shape, w["embed"][5], k, v, keep | (at == n) if bool(keep[n]) else keep)
                assert bool(((wrong - want).abs() > 2 * tol).any()), (n, int(keep.sum()))


# (hd, kv heads, group, sequences, max_context, longest): on 256 CUs
CASES = [
    (128, 2, 4, 2, 3008, 3000), (64, 2, 4, 2, 3008, 3000), (128, 1, 8, 3, 6000, 5990), (64, 2, 3, 3, 4096, 4090),     # 6 - 12 parts of 8 steps
    (128, 2, 4, 150, 8000, 7900), (64, 2, 4, 150, 8000, 7900),                                                      # 2 parts, more workgroups than CUs
    (128, 2, 4, 16, 65536, 20000), (64, 2, 4, 16, 131072, 9000),                                                    # parts, past the caches
    (128, 2, 4, 96, 1024, 1020), (64, 2, 4, 96, 1024, 1020), (128, 1, 8, 200, 900, 890),                            # whole, by eight waves
    (128, 2, 4, 96, 16384, 5000), (64, 2, 4, 96, 32768, 5000),                                                      # ... past the caches
    (128, 2, 4, 260, 4096, 1500), (64, 2, 4, 260, 8192, 1500),                                                      # whole, by four, past the caches
    (128, 2, 4, 200, 512, 500), (64, 2, 3, 140, 300, 290),                                                          # whole, by four
]


@pytest.mark.gpu
@pytest.mark.parametrize("hd,kv_heads,group,num,max_context,longest", CASES)
def test_attention_of_the_decoding_step(hd, kv_heads, group, num, max_context, longest):
    shape, w = mirror_model(kv_heads, group, hd)
    sess = VerifierSession(shape, w, max_position=max_context, device=DEV)
    g, rng = torch.Generator().manual_seed(num + hd), wl.rng_for(num, hd)
    few = [longest - 1, longest - 16 + longest % 16, longest - 64]                     # (the last of a block, the first, some other)
    lens = (few + [n for n in BORDERS if n < longest])[:num]
    lens += [int(x) for x in rng.integers(0, min(longest, 700), num - len(lens))]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=2, max_blocks_per_seq=-(-max_context // 16))
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    cached = []
    for s, n in enumerate(lens):
        k, v = cached_kv(shape, n, g)
        cached.append((k, v))
        if n:
            both = [torch.cat((t[None], torch.zeros(group, *t.shape, dtype=t.dtype))) for t in (k, v)]
            kv_layout.write_tokens(kv, bt[s], *both)
    seq, tok = i32(lens), i32(rng.integers(0, VOCAB, num))
    kv4 = sess.kv4_cache(blocks)
    kv4.fill_(255)                                                                    # (NaN wherever nothing was stored)
    sess.kv4_store(kv, kv4, bt, torch.zeros_like(seq), seq, max(lens))
    stored, status = kv4.clone(), i32([9] * num)
    out = sess.decode_mx4(kv, bt, seq, tok, kv4, max_context=max_context, seq_status=status).clone()
    assert not bool(status.any())
    # the newest position, as the attention kernel stored it, in every layer, and no other byte
    sess.kv4_store(kv, stored, bt, seq, torch.ones_like(seq), 1)
    assert torch.equal(kv4, stored)
    for s, n in enumerate(lens):
        k, v = kv_layout.read_tokens(kv, bt[s], n + 1, hd)
        k, v = k[:, n].cpu(), v[:, n].cpu()
        want, tol = normed(shape, w["embed"][int(tok[s])], torch.cat((cached[s][0], k[:1])), torch.cat((cached[s][1], v[:1])))
        err = (v[1:].flatten().double() - want).abs()
        assert bool((err <= tol).all()), (s, n, float((err / tol).max()))
    # the same call gives the same bits
    before = kv.clone()
    assert torch.equal(sess.decode_mx4(kv, bt, seq, tok, kv4, max_context=max_context), out)
    assert torch.equal(kv4, stored) and torch.equal(kv, before)
    sess.close()


@pytest.mark.gpu
@pytest.mark.parametrize("num", [1, 5, 24, 90])
@pytest.mark.parametrize("four_bit_cache", [False, True], ids=["bf16_cache", "4bit_cache"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_a_repeated_step_gives_the_same_tokens(num, four_bit_cache, temperature):
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=256, device=DEV)
    rng = wl.rng_for(5, num)
    lens = [int(x) for x in rng.integers(1, 120, num)]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    kv4 = sess.kv4_cache(blocks) if four_bit_cache else None
    if four_bit_cache:
        sess.kv4_store(kv, kv4, bt, i32([0] * num), i32(lens), max(lens))
    sampling = B.make_sampling(temperature, 77, torch.arange(num, device=DEV)) if temperature else None
    step = lambda: sess.decode_mx4(kv, bt, i32(lens), tok, kv4, sampling=sampling)
    want = step()
    assert all(torch.equal(step(), want) for _ in range(3))
    sess.close()
