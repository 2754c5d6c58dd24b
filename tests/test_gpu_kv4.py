"""The 4-bit cache on the GPU: storing and reading it bit for bit, attention over it against float64, the fast path that runs on it."""
import ctypes
import json
import math

import numpy as np
import pytest
import torch

import mx4_reference as ref
from gpu_helpers import NOISE_FACTOR
from helpers import orc, wl, oracle_cfg, randomize_gains
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd import dvr, dvr_stats, kv_layout
from paper_2601_17768_amd.mx4 import Mx4Matrix
from paper_2601_17768_amd.session import VerifierSession

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


def session(kv_heads=2, group=2, hd=64, layers=2):
    shape = wl.ModelShape(n_layers=layers, d_model=128, n_q_heads=kv_heads * group, n_kv_heads=kv_heads, head_dim=hd, d_ffn=64, vocab=16,
                          rope_theta=1e4)
    return VerifierSession(shape, wl.make_weights(shape), max_position=16384, device=DEV)


class Cache:
    """K and V of some sequences, in a bf16 paged cache and beside it."""

    def __init__(self, sess, lens, seed=0, width=None):
        s, g = sess.shape, torch.Generator().manual_seed(seed)
        self.lens = [int(n) for n in lens]
        table, blocks = wl.make_block_table(wl.rng_for(seed, 5), [max(n, 1) for n in self.lens], 16, spare_blocks=3, max_blocks_per_seq=width)
        self.bt, self.kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
        self.k, self.v = [], []
        for i, n in enumerate(self.lens):
            k, v = (torch.randn(s.n_layers, n, s.n_kv_heads, s.head_dim, generator=g) for _ in range(2))
            k = (k * torch.exp2(torch.randint(-3, 4, (s.n_kv_heads, s.head_dim), generator=g).float())).to(torch.bfloat16)
            v = (v * torch.exp2(torch.randint(-6, 7, (n, 1, 1), generator=g).float())).to(torch.bfloat16)
            self.k.append(k)
            self.v.append(v)
            if n:
                kv_layout.write_tokens(self.kv, self.bt[i], k, v)

    def mirror(self, sess):
        """A 4-bit cache whose every other byte is 0xFF: scales of NaN wherever nothing was stored."""
        kv4 = sess.kv4_cache(self.kv.shape[2])
        kv4.fill_(255)
        sess.kv4_store(self.kv, kv4, self.bt, i32([0] * len(self.lens)), i32(self.lens), max(max(self.lens), 1))
        return kv4


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kv_heads", [1, 3, 8])
def test_store_and_read(hd, kv_heads):
    sess = session(kv_heads, 1, hd, layers=3)
    c = Cache(sess, [1, 16, 17, 40, 100, 33, 0])
    c.v[4][0, 50, 0, 3] = float("inf")
    c.k[4][1, 51, 0, hd - 1] = float("nan")
    kv_layout.write_tokens(c.kv, c.bt[4], c.k[4], c.v[4])
    kv4 = sess.kv4_cache(c.kv.shape[2])
    kv4.fill_(0x5A)
    first, count = [0, 3, 5, 0, 17, 32, 0], [1, 9, 12, 40, 66, 1, 0]
    status = i32([9] * 7)
    sess.kv4_store(c.kv, kv4, c.bt, i32(first), i32(count), 70, seq_status=status)
    assert status.tolist() == [0] * 7
    ok, ov = (torch.full((3, 7, 70, kv_heads, hd), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    status.fill_(9)
    sess.kv4_read(kv4, c.bt, i32(first), i32(count), 70, ok, ov, seq_status=status)
    assert status.tolist() == [0] * 7
    for got, plain in ((ok, c.k), (ov, c.v)):
        for s in range(7):
            want = ref.quantized(plain[s][:, first[s]:first[s] + count[s]])
            have = got[:, s, :count[s]].cpu().double()
            assert torch.equal(torch.isnan(have), torch.isnan(want)) and torch.equal(torch.nan_to_num(have), torch.nan_to_num(want))
            assert bool((got[:, s, count[s]:] == 5.0).all())
    sess.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_store_leaves_every_other_position_alone(hd):
    """Position by position, in any order, gives what one call gives; what was never stored keeps its bytes."""
    sess = session(2, 1, hd)
    c = Cache(sess, [37, 20])
    whole = c.mirror(sess)
    parts = sess.kv4_cache(c.kv.shape[2])
    parts.fill_(255)
    for p in np.random.default_rng(1).permutation(37):
        sess.kv4_store(c.kv, parts, c.bt, i32([p, min(p, 19)]), i32([1, 1 if p < 20 else 0]), 1)
    assert torch.equal(whole, parts)
    used = set(c.bt[0, :3].tolist()) | set(c.bt[1, :2].tolist())
    spare = [b for b in range(c.kv.shape[2]) if b not in used]
    assert bool((whole[:, spare] == 255).all())
    sess.close()


def test_store_and_read_flag_sequences_and_leave_them_out():
    sess = session()
    c = Cache(sess, [40] * 6, width=4)
    kv4 = sess.kv4_cache(c.kv.shape[2])
    kv4.fill_(255)
    bt = c.bt.clone()
    bt[4, 1] = c.kv.shape[2]
    bt[5, 2] = -1
    first, count = [-1, 0, 60, 8, 8, 8], [1, 41, 5, 20, 20, 20]
    status = i32([9] * 6)
    sess.kv4_store(c.kv, kv4, bt, i32(first), i32(count), 40, seq_status=status)
    L, K, OK = B.LLM42_SEQ_BAD_LENGTH, B.LLM42_SEQ_BAD_BLOCK, 0
    assert status.tolist() == [L, L, L, OK, K, OK]               # (the last one's entry is not among those it needs)
    for s in (0, 1, 2, 4):
        assert bool((kv4[:, c.bt[s, :3].long()] == 255).all())
    status.fill_(9)
    ok, ov = sess.kv4_read(kv4, bt, i32(first), i32(count), 40, seq_status=status)
    assert status.tolist() == [L, L, L, OK, K, OK]
    assert all(bool((x[:, s] == 0).all()) for x in (ok, ov) for s in (0, 1, 2, 4))
    # a table of its own for the 4-bit cache is checked as well, and a status is not asked for
    bt4 = c.bt.clone()
    bt4[3, 1] = -7
    kv4.fill_(255)
    sess.kv4_store(c.kv, kv4, c.bt, i32(first), i32(count), 40, kv4_block_table=bt4, seq_status=status)
    assert status.tolist() == [L, L, L, K, OK, OK]
    sess.kv4_store(c.kv, kv4, c.bt, i32(first), i32(count), 40, kv4_block_table=bt4)
    assert bool((kv4[:, c.bt[3, :3].long()] == 255).all())
    sess.close()


def check_attention(sess, lens, n_valid, window, max_context=None, seed=3, layer=1):
    """lens: cached before the window.  Every weight is rounded to bf16 once (2^-8 of it at most), the output once, exp2 and the
    fp32 sums stay far below that."""
    s = sess.shape
    rows = [window] * len(lens) if n_valid is None else n_valid
    c = Cache(sess, [a + b for a, b in zip(lens, rows)], seed)
    kv4 = c.mirror(sess)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(len(lens), window, s.n_q_heads, s.head_dim, generator=g).to(torch.bfloat16)
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device=DEV)
    status = i32([9] * len(lens))
    got = sess.kv4_attention(layer, kv4, c.bt, q.to(DEV), i32(lens), None if n_valid is None else i32(n_valid), max_context, out, status).cpu()
    assert status.tolist() == [0] * len(lens)
    for i, (a, n) in enumerate(zip(lens, rows)):
        assert bool((got[i, n:] == 5.0).all())
        if n:
            want, mag = ref.attention(q[i, :n].double(), ref.quantized(c.k[i][layer]), ref.quantized(c.v[i][layer]), a)
            tol = 2.0 ** -8 * mag + 2.0 ** -8 * want.abs() + 2.0 ** -14 * mag
            err = (got[i, :n].double() - want).abs()
            assert bool((err <= tol).all()), (i, a, n, float((err / tol).max()))
    return c, kv4, q


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 8])
def test_attention_of_single_tokens(hd, group):
    sess = session(2, group, hd)
    check_attention(sess, [0, 1, 14, 15, 16, 62, 63, 64, 65, 255, 256, 500, 1000], None, 1)
    check_attention(sess, [5], None, 1)
    check_attention(sess, [2500], None, 1, max_context=2501)
    sess.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("group,window", [(1, 2), (2, 13), (4, 4), (4, 8), (8, 5), (3, 11), (4, 32), (7, 64), (1, 100)])
def test_attention_of_windows(hd, group, window):
    sess = session(2, group, hd)
    check_attention(sess, [0, 1, 63, 130, 700], None, window)
    ragged = [window, 0, 1, max(1, window // 2), max(1, window - 1)]
    check_attention(sess, [300, 40, 0, 64, 1100], ragged, window)
    sess.close()


def test_attention_of_many_sequences_and_one_part():
    sess = session(8, 4, 128, layers=2)
    check_attention(sess, [int(n) for n in np.random.default_rng(0).integers(0, 300, 150)], None, 1)
    sess.close()


def test_attention_of_rows_apart_and_of_flagged_sequences():
    sess = session(2, 2, 64)
    c = Cache(sess, [50, 50, 50, 50], width=5)
    kv4 = c.mirror(sess)
    q = torch.randn(4, 3, 4, 64, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).to(DEV)
    lens = i32([47, 47, 47, 47])
    want = sess.kv4_attention(0, kv4, c.bt, q, lens)
    wide = torch.full((4, 3, 6, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    wide[:, :, :4] = q
    got = torch.full((4, 3, 5, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    sess.kv4_attention(0, kv4, c.bt, wide[:, :, :4], lens, out=got[:, :, :4])
    assert torch.equal(got[:, :, :4], want) and bool((got[:, :, 4] == 9.0).all())
    bt = c.bt.clone()
    bt[1, 2] = -1
    bt[3, 4] = -1                                                # beyond what the sequence needs
    status, out = i32([9] * 4), torch.full_like(q, 9.0)
    sess.kv4_attention(0, kv4, bt, q, i32([47, 47, 78, 47]), i32([3, 3, 3, 3]), 80, out, status)
    assert status.tolist() == [0, B.LLM42_SEQ_BAD_BLOCK, B.LLM42_SEQ_BAD_LENGTH, 0]
    assert torch.equal(out[0], want[0]) and torch.equal(out[3], want[3]) and bool((out[1:3] == 9.0).all())
    for n_valid, lens2 in (([4, 3, 3, 3], [47] * 4), ([-1, 3, 3, 3], [47] * 4), ([3] * 4, [-1, 47, 47, 47])):
        sess.kv4_attention(0, kv4, c.bt, q, i32(lens2), i32(n_valid), 80, out, status)
        assert status.tolist() == [B.LLM42_SEQ_BAD_LENGTH, 0, 0, 0]
    for kwargs, code in ((dict(layer=2), B.LLM42_EINVAL), (dict(layer=-1), B.LLM42_EINVAL), (dict(max_context=81), B.LLM42_ECAPACITY)):
        a = {**dict(layer=0, max_context=80), **kwargs}
        with pytest.raises(B.Llm42Error) as e:
            sess.kv4_attention(a["layer"], kv4, c.bt, q, lens, None, a["max_context"], out)
        assert e.value.status == code
    for bad in (q.transpose(1, 2), q.float(), q[:, :, :, :32], q[:2]):
        with pytest.raises(ValueError):
            sess.kv4_attention(0, kv4, c.bt, bad, lens, out=torch.zeros_like(bad))
    for few in (q[:, :, :2], q[:, :, :2].contiguous()):          # rows of fewer heads than the model has
        with pytest.raises(ValueError):
            sess.kv4_attention(0, kv4, c.bt, few, lens)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    with pytest.raises(B.Llm42Error):
        B.llm42_kv4_attention(sess.model, 0, kv4, kv4.shape[1], c.bt, q[:, :, :2].contiguous(), lens, None, 80, torch.zeros_like(q[:, :, :2]), ws)
    sess.close()


def test_attention_store_and_read_refuse_at_the_c_entry():
    """Addresses are real, so that a call which were not refused would be harmless."""
    lib, sess = B.load_library(), session(2, 2, 64)
    c = Cache(sess, [50, 50])
    kv4, q, lens = c.mirror(sess), torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device=DEV), i32([10, 10])
    need = B.llm42_kv4_attention_workspace_bytes(sess.model, 2, 3, 64)
    ws = torch.empty(need + 512, dtype=torch.uint8, device=DEV)
    view = lambda **k: B.KVCache(*{**dict(base=kv4.data_ptr(), blocks=kv4.shape[1], table=c.bt.data_ptr(), width=4), **k}.values())
    kv = lambda **k: view(**{**dict(base=c.kv.data_ptr()), **k})
    p = lambda t, off=0: t.data_ptr() + off
    base = dict(model=sess.model, layer=0, kv4=view(), q=p(q), qs=256, lens=p(lens), window=3, valid=None, num=2, ctx=64, out=p(q), os=256,
                status=None, ws=p(ws), bytes=need, stream=None)
    for bad, code in [(dict(model=None), B.LLM42_EINVAL), (dict(layer=2), B.LLM42_EINVAL), (dict(q=None), B.LLM42_EINVAL),
                      (dict(out=None), B.LLM42_EINVAL), (dict(lens=None), B.LLM42_EINVAL), (dict(ws=None), B.LLM42_EINVAL),
                      (dict(q=p(q, 8)), B.LLM42_EINVAL), (dict(out=p(q, 2)), B.LLM42_EINVAL), (dict(qs=255), B.LLM42_EINVAL),
                      (dict(qs=260), B.LLM42_EINVAL), (dict(os=248), B.LLM42_EINVAL), (dict(window=0), B.LLM42_EINVAL),
                      (dict(window=B.LLM42_MAX_WINDOW + 1), B.LLM42_EINVAL), (dict(num=0), B.LLM42_EINVAL),
                      (dict(num=B.LLM42_MAX_ROWS // 3 + 1), B.LLM42_EINVAL), (dict(ctx=0), B.LLM42_EINVAL), (dict(ctx=65), B.LLM42_ECAPACITY),
                      (dict(ctx=2 ** 30 + 1), B.LLM42_EINVAL), (dict(ws=p(ws, 16)), B.LLM42_EWORKSPACE), (dict(bytes=need - 1), B.LLM42_EWORKSPACE),
                      (dict(kv4=view(base=None)), B.LLM42_EINVAL), (dict(kv4=view(base=kv4.data_ptr() + 8)), B.LLM42_EINVAL),
                      (dict(kv4=view(table=None)), B.LLM42_EINVAL), (dict(kv4=view(blocks=0)), B.LLM42_EINVAL), (dict(kv4=view(width=0)), B.LLM42_EINVAL)]:
        a = {**base, **bad}
        a["kv4"] = ctypes.byref(a["kv4"])
        assert lib.llm42_kv4_attention(*a.values()) == code, bad
    base = dict(model=sess.model, kv=kv(), kv4=view(), first=p(lens), count=p(lens), num=2, most=64, status=None, stream=None)
    for bad in (dict(model=None), dict(first=None), dict(count=None), dict(num=0), dict(most=0), dict(num=2 ** 31 - 1, most=2 ** 31 - 1),
                dict(kv=kv(base=None)), dict(kv=kv(table=None)), dict(kv4=view(base=None)), dict(kv4=view(blocks=0))):
        a = {**base, **bad}
        assert lib.llm42_kv4_store(a["model"], ctypes.byref(a["kv"]), ctypes.byref(a["kv4"]), *list(a.values())[3:]) == B.LLM42_EINVAL, bad
        if "kv" not in bad:
            out = torch.zeros(2 * 2 * 64 * 2 * 64, dtype=torch.bfloat16, device=DEV)
            assert lib.llm42_kv4_read(a["model"], ctypes.byref(a["kv4"]), a["first"], a["count"], a["num"], a["most"], p(out), p(out), None,
                                      None) == B.LLM42_EINVAL, bad
    out = torch.zeros(2 * 2 * 64 * 2 * 64, dtype=torch.bfloat16, device=DEV)
    for k, v in ((None, p(out)), (p(out), None), (p(out, 8), p(out))):
        assert lib.llm42_kv4_read(sess.model, ctypes.byref(view()), p(lens), p(lens), 2, 64, k, v, None, None) == B.LLM42_EINVAL
    m4, size = sess.mx4, ctypes.c_size_t()
    assert lib.llm42_decode_step_mx4_workspace_bytes(m4, 2, 64, None) == B.LLM42_EINVAL
    assert lib.llm42_decode_step_mx4_workspace_bytes(m4, 0, 64, ctypes.byref(size)) == B.LLM42_EINVAL
    assert lib.llm42_mx4_model_create(sess.model, None) == B.LLM42_EINVAL
    assert lib.llm42_decode_step_mx4_workspace_bytes(m4, 2, 64, ctypes.byref(size)) == B.LLM42_OK
    need = size.value
    ws, tok = torch.empty(need + 512, dtype=torch.uint8, device=DEV), i32([1, 1])
    base = dict(m4=m4, kv=kv(), kv4=view(), lens=p(lens), tok=p(tok), num=2, ctx=64, out=p(tok), status=None, ws=p(ws), bytes=need, stream=None,
                sampling=None)
    for bad, code in [(dict(m4=None), B.LLM42_EINVAL), (dict(lens=None), B.LLM42_EINVAL), (dict(tok=None), B.LLM42_EINVAL), (dict(out=None), B.LLM42_EINVAL),
                      (dict(num=0), B.LLM42_EINVAL), (dict(ctx=65), B.LLM42_ECAPACITY), (dict(kv4=view(width=3)), B.LLM42_ECAPACITY),
                      (dict(kv4=view(base=None)), B.LLM42_EINVAL), (dict(kv4=view(table=None)), B.LLM42_EINVAL), (dict(kv=kv(base=None)), B.LLM42_EINVAL),
                      (dict(ws=p(ws, 128)), B.LLM42_EWORKSPACE), (dict(bytes=4096), B.LLM42_EWORKSPACE),
                      (dict(sampling=ctypes.byref(B.Sampling(-1.0, 0, None))), B.LLM42_EINVAL)]:
        a = {**base, **bad}
        a["kv"], a["kv4"] = ctypes.byref(a["kv"]), ctypes.byref(a["kv4"])
        assert lib.llm42_decode_step_mx4(*a.values()) == code, bad
    torch.cuda.synchronize()
    sess.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_rows_do_not_see_a_later_nan(hd):
    """A NaN in K or V of one position of the window: the rows before it keep their bits, those from it on have the NaN - of V only in the
    32 features that share its scale.  (Behind 3000 positions in parts, and at every place in a step of keys.)"""
    sess = session(2, 4, hd)
    lens, window = [0, 50, 60, 63, 64, 3000], 13
    c, kv4, q = check_attention(sess, lens, None, window)
    qd, at = q.to(DEV), 5
    clean = sess.kv4_attention(1, kv4, c.bt, qd, i32(lens))
    for which, value in (("k", math.nan), ("v", math.nan), ("v", math.inf), ("k", -math.inf)):
        for i, a in enumerate(lens):
            k, v = c.k[i].clone(), c.v[i].clone()
            (k if which == "k" else v)[1, a + at, 1, 33] = value
            kv_layout.write_tokens(c.kv, c.bt[i], k, v)
        got = sess.kv4_attention(1, c.mirror(sess), c.bt, qd, i32(lens))
        assert torch.equal(got[:, :at], clean[:, :at]) and torch.equal(got[:, at:, :4], clean[:, at:, :4])
        nan = torch.isnan(got[:, at:, 4:])
        if which == "k":
            assert bool(nan.all())
        else:
            assert bool(nan[..., 32:64].all()) and not bool(nan[..., :32].any()) and not bool(nan[..., 64:].any())
            assert torch.equal(got[:, at:, 4:, :32], clean[:, at:, 4:, :32]) and torch.equal(got[:, at:, 4:, 64:], clean[:, at:, 4:, 64:])
    sess.close()


def test_attention_of_the_longest_window_and_the_most_sequences():
    sess = session(2, 8, 64)
    check_attention(sess, [0, 700], [B.LLM42_MAX_WINDOW, 500], B.LLM42_MAX_WINDOW)
    c = Cache(sess, [33, 20])
    kv4, num = c.mirror(sess), B.LLM42_MAX_ROWS                  # (as many as a call takes, on the blocks of two)
    q = torch.randn(num, 1, 16, 64, device=DEV).to(torch.bfloat16)
    lens = i32([32, 19]).repeat(num // 2)
    got = sess.kv4_attention(1, kv4, c.bt.repeat(num // 2, 1), q, lens)
    for at in (0, 31000, num - 2):                               # (one step of keys: the same sums alone)
        assert torch.equal(got[at:at + 2], sess.kv4_attention(1, kv4, c.bt, q[at:at + 2].contiguous(), lens[:2].contiguous()))
    sess.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_store_and_read_of_many_sequences_and_in_a_graph(hd):
    sess = session(3, 2, hd)
    c, num = Cache(sess, [40]), 30000                            # every sequence reads the one cache; the first of them stores
    kv4 = c.mirror(sess)
    first, count = i32([7] * num), i32([0] * (num - 1) + [30])
    k, v = sess.kv4_read(kv4, c.bt.repeat(num, 1), first, count, 30)
    assert torch.equal(k[:, -1].cpu(), ref.quantized(c.k[0][:, 7:37]).to(torch.bfloat16))
    assert torch.equal(v[:, -1].cpu(), ref.quantized(c.v[0][:, 7:37]).to(torch.bfloat16)) and not bool(k[:, :-1].any())
    status = i32([9] * num)
    kv4.fill_(255)
    sess.kv4_store(c.kv, kv4, c.bt.repeat(num, 1), first, count, 30, seq_status=status)
    assert not bool(status.any())
    a, n = i32([0]), i32([40])
    ko, vo = (torch.zeros(2, 1, 40, 3, hd, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    sess.kv4_store(c.kv, kv4, c.bt, a, n, 40)
    with torch.cuda.graph(graph):
        sess.kv4_store(c.kv, kv4, c.bt, a, n, 40)
        sess.kv4_read(kv4, c.bt, a, n, 40, ko, vo)
    for lo, cnt, scale in ((0, 40, 1.0), (16, 16, 2.0), (39, 1, -0.5), (3, 0, 4.0), (5, 30, 1.0)):
        before = sess.kv4_read(kv4, c.bt, i32([0]), i32([40]), 40)
        kv_layout.write_tokens(c.kv, c.bt[0], c.k[0] * scale, c.v[0] * scale)
        a.fill_(lo), n.fill_(cnt), ko.fill_(1.0), vo.fill_(1.0)
        graph.replay()
        after = sess.kv4_read(kv4, c.bt, i32([0]), i32([40]), 40)
        for x, out, old, new in ((c.k[0], ko, before[0], after[0]), (c.v[0], vo, before[1], after[1])):
            want = ref.quantized(x * scale).to(torch.bfloat16)[:, lo:lo + cnt]
            assert torch.equal(out[:, 0, :cnt].cpu(), want) and bool((out[:, 0, cnt:] == 1.0).all())
            old[:, 0, lo:lo + cnt] = want.to(DEV)
            assert torch.equal(new, old)
    sess.close()


def test_attention_of_empty_windows_in_parts():
    sess = session(2, 4, 128)
    check_attention(sess, [5000, 0, 4000, 77], [0, 0, 1, 3], 5)
    check_attention(sess, [5000, 0], [0, 0], 1)
    sess.close()


def test_a_cache_of_more_than_4_gib():
    """Blocks at both ends of it, and their offsets beyond 32 bits."""
    sess = session(8, 4, 128, layers=1)
    c = Cache(sess, [40, 100])
    blocks = 260000
    kv, kv4 = torch.empty((1, 2, blocks) + tuple(c.kv.shape[3:]), dtype=torch.bfloat16, device=DEV), sess.kv4_cache(blocks)
    assert kv4.numel() > 2 ** 32 and kv.shape[3:] == c.kv.shape[3:] and c.kv.shape[2] < 200
    far = c.bt.clone()
    far[c.bt >= 5] += blocks - c.kv.shape[2]
    kv[:, :, :5] = c.kv[:, :, :5]
    kv[:, :, 5 + blocks - c.kv.shape[2]:] = c.kv[:, :, 5:]
    near, n = c.mirror(sess), i32([40, 100])
    sess.kv4_store(kv, kv4, far, i32([0, 0]), n, 100)
    for a, b in zip(sess.kv4_read(kv4, far, i32([0, 0]), n, 100), sess.kv4_read(near, c.bt, i32([0, 0]), n, 100)):
        assert torch.equal(a, b)
    q = torch.randn(2, 1, 32, 128, device=DEV).to(torch.bfloat16)
    assert torch.equal(sess.kv4_attention(0, kv4, far, q, n - 1), sess.kv4_attention(0, near, c.bt, q, n - 1))
    sess.close()


def test_calls_stay_within_their_workspace():
    sess = session(2, 4, 64)
    c = Cache(sess, [3000, 20])
    kv4, q, lens = c.mirror(sess), torch.randn(2, 7, 8, 64, device=DEV).to(torch.bfloat16), i32([2993, 13])
    need = B.llm42_kv4_attention_workspace_bytes(sess.model, 2, 7, 3008)
    assert need > 2 * 7 * 8 * 64 * 4                             # (in parts)
    ws, out = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV), torch.zeros_like(q)
    B.llm42_kv4_attention(sess.model, 0, kv4, kv4.shape[1], c.bt, q, lens, None, 3008, out, ws[:need])
    assert bool((ws[need:] == 77).all()) and torch.equal(out, sess.kv4_attention(0, kv4, c.bt, q, lens, max_context=3008))
    for num in (1, 2):
        need = B.llm42_decode_step_mx4_workspace_bytes(sess.mx4, num, 3008)
        ws, nxt = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV), i32([0] * num)
        for cache in (None, kv4):
            B.llm42_decode_step_mx4(sess.model, sess.mx4, c.kv, c.kv.shape[2], c.bt[:num].contiguous(), cache, kv4.shape[1], c.bt[:num].contiguous(),
                                    lens[:num].contiguous(), i32([3] * num), 3008, nxt, ws[:need])
            assert bool((ws[need:] == 77).all())
    sess.close()


def test_two_graphs_of_one_session_and_a_workspace_that_is_outgrown():
    sess = session(2, 4, 128)
    c = Cache(sess, [900, 40])
    kv4, q = c.mirror(sess), torch.randn(2, 4, 8, 128, device=DEV).to(torch.bfloat16)
    lens = i32([800, 30])
    want = [sess.kv4_attention(0, kv4, c.bt, q[:, :w].contiguous(), lens) for w in (1, 4)]
    sess._ws = None                                              # (the first capture makes it)
    graphs, outs, inputs = [], [], []
    for w in (1, 4):
        graphs.append(torch.cuda.CUDAGraph())
        inputs.append(q[:, :w].contiguous())
        outs.append(torch.zeros_like(inputs[-1]))
        with torch.cuda.graph(graphs[-1]):
            sess.kv4_attention(0, kv4, c.bt, inputs[-1], lens, out=outs[-1])
    sess.kv4_attention(0, kv4, c.bt, q.repeat(1, 60, 1, 1), i32([600, 20]), i32([240, 10]))
    others = [torch.full((1 << 22,), float(i), device=DEV) for i in range(8)]
    for i in (0, 1, 1, 0, 1, 0):
        outs[i].fill_(2.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])
    assert all(bool((t == float(i)).all()) for i, t in enumerate(others))
    with pytest.raises(RuntimeError):                            # the model's 4-bit copy cannot be made inside a capture
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            sess.decode_mx4(c.kv, c.bt, lens, i32([1, 1]))
    del graphs
    torch.cuda.synchronize()
    sess.close()


def test_attention_weights_of_large_and_masked_scores():
    """Scores of +-1e4, keys that are all alike, and one key that takes everything."""
    sess = session(1, 4, 128, layers=1)
    n = 300
    c = Cache(sess, [n])
    for what in ("spike", "alike", "large"):
        k, v = torch.zeros(1, n, 1, 128), torch.randn(1, n, 1, 128, generator=torch.Generator().manual_seed(2))
        if what == "spike":
            k[0, 170, 0, :] = 400.0
        if what == "large":
            k[:] = torch.randn(1, n, 1, 128, generator=torch.Generator().manual_seed(4)) * 300
        c.k[0], c.v[0] = k.to(torch.bfloat16), v.to(torch.bfloat16)
        kv_layout.write_tokens(c.kv, c.bt[0], c.k[0], c.v[0])
        kv4 = c.mirror(sess)
        q = torch.ones(1, 1, 4, 128, dtype=torch.bfloat16)
        got = sess.kv4_attention(0, kv4, c.bt, q.to(DEV), i32([n - 1])).cpu().double()
        want, mag = ref.attention(q[0].double(), ref.quantized(c.k[0][0]), ref.quantized(c.v[0][0]), n - 1)
        # (a score of size S carries an error of 128 S 2^-23 from its sum, which the exponential passes on)
        slack = 128 * 2.0 ** -23 * (float(ref.quantized(c.k[0][0]).abs().sum(-1).max()) * 128 ** -0.5) * 2
        # (a weight below 2^-126 of the largest has no normal fp32 and may count as 0: off by less than 2^-126 |v| for each of the n keys)
        under = n * 2.0 ** -126 * float(c.v[0].abs().max()) * 2
        fine = (got[0] - want).abs() <= (2.0 ** -7 + 2.0 ** -14 + slack) * mag + 2.0 ** -8 * want.abs() + under
        assert bool(fine.all()), what
    sess.close()


def test_attention_in_a_graph_and_on_another_stream():
    sess = session(2, 4, 128)
    c, kv4, q = check_attention(sess, [100, 600, 3], None, 1)
    qd, lens = q.to(DEV), i32([100, 600, 3])
    want = sess.kv4_attention(0, kv4, c.bt, qd, lens)
    out = torch.zeros_like(want)
    sess.kv4_attention(0, kv4, c.bt, qd, lens, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sess.kv4_attention(0, kv4, c.bt, qd, lens, out=out)
    for cut in (0, 50, 3):
        lens.copy_(i32([100 - cut, 600 - cut, 3 - min(cut, 3)]))
        want = sess.kv4_attention(0, kv4, c.bt, qd, lens)
        out.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = sess.kv4_attention(0, kv4, c.bt, qd, lens)
    torch.cuda.synchronize()
    assert torch.equal(other, want)
    sess.close()


# ---- the fast path ----------------------------------------------------------------------------------------------
HEADS128 = wl.ModelShape(n_layers=2, d_model=256, n_q_heads=6, n_kv_heads=2, head_dim=128, d_ffn=336, vocab=512, rope_theta=1e4)


@pytest.mark.parametrize("shape", [wl.TINY, HEADS128], ids=["hd64", "hd128"])
@pytest.mark.parametrize("four_bit_cache", [False, True], ids=["bf16_cache", "4bit_cache"])
def test_decode_step_against_the_oracle_on_the_quantised_model(shape, four_bit_cache):
    """The oracle run on the weights that the 4-bit copy stands for, with a cache that holds what the 4-bit one does: the same token
    wherever its two best logits are further apart than twice the small model's tolerance."""
    w = randomize_gains(wl.make_weights(shape, seed=11))
    cfg, wq = oracle_cfg(shape), ref.quantized_weights(w)
    sess = VerifierSession(shape, w, max_position=512, device=DEV)
    rng = wl.rng_for(11, 3)
    lens = [1, 7, 16, 40, 130, 64, 15, 3, 90, 33, 5, 18, 77, 21, 31, 47, 2, 63, 100, 12]
    prompts = [wl.random_tokens(rng, n, shape.vocab) for n in lens]
    table, blocks = wl.make_block_table(rng, [n + 4 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, prompts, window=16)
    kv4 = None
    if four_bit_cache:
        kv4 = sess.kv4_cache(blocks)
        kv4.fill_(255)
        sess.kv4_store(kv, kv4, bt, i32([0] * len(lens)), i32(lens), max(lens))
    caches = []
    for s, n in enumerate(lens):                                  # the verifier's K and V, as the step finds them
        k, v = kv_layout.read_tokens(kv, bt[s], n, shape.head_dim)
        okv = ref.QuantizingKV(cfg, n + 4) if four_bit_cache else orc.OracleKV(cfg, n + 4)
        okv.k[:, :n], okv.v[:, :n] = k.cpu().double(), v.cpu().double()
        caches.append(okv)
    seq, status, decided = i32(lens), i32([9] * len(lens)), 0
    for step in range(3):
        nxt = sess.decode_mx4(kv, bt, seq, tok, kv4, seq_status=status)
        assert status.tolist() == [0] * len(lens)
        for s, n in enumerate(lens):
            logits = orc.forward_window(cfg, wq, caches[s], n + step, [int(tok[s])])
            if float(orc.top2_margin(logits)[0]) > 4e-2:
                assert int(nxt[s]) == int(orc.greedy_argmax(logits)[0]), (step, s)
                decided += 1
        seq += 1
        tok = nxt.clone()
    assert decided >= 30, decided
    sess.close()

@pytest.mark.parametrize("num", [1, 8, 24, 128])
def test_decode_step_at_the_8b_widths_is_the_model_of_the_quantised_values(num):
    """Two layers: the step's token is a best one of the verifier on the weights that the 4-bit copy stands for, up to the logits' rounding
    (both round the same operands to bf16, and differ in the order of their sums: an error of up to 3.5e-2 at these widths and two layers,
    gpu_helpers.py, times its NOISE_FACTOR, for each of the two logits compared)."""
    shape = wl.LLAMA_8B.replace(n_layers=2, vocab=16384)
    to = lambda w, f: {"embed": w["embed"].to(DEV), "final_norm": w["final_norm"].to(DEV), "lm_head": f(w["lm_head"].to(DEV)),
                       "layers": [{n: t.to(DEV) if n.endswith("norm") else f(t.to(DEV)) for n, t in lw.items()} for lw in w["layers"]]}
    w = wl.make_weights(shape, seed=42)
    sess = VerifierSession(shape, to(w, lambda t: t), max_position=1024, device=DEV)
    values = VerifierSession(shape, to(w, lambda t: Mx4Matrix.quantize(t).values()), max_position=1024, device=DEV)
    rng = wl.rng_for(5, num)
    lens = [int(n) for n in rng.integers(1, 400, num)]
    table, blocks = wl.make_block_table(rng, [n + 2 for n in lens], 16, spare_blocks=2)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=64)
    copy = kv.clone()
    got = sess.decode_mx4(kv, bt, i32(lens), tok)
    logits = torch.empty((num, 1, shape.vocab), dtype=torch.float32, device=DEV)
    values.verify(copy, bt, i32(lens), tok.view(num, 1), dump_seq_ids=i32(range(num)), out_logits=logits)
    gap = logits[:, 0].max(1).values - logits[:, 0].gather(1, got.long().view(num, 1))[:, 0]
    assert float(gap.max()) <= 2 * NOISE_FACTOR * 3.5e-2, gap
    sess.close()
    values.close()


@pytest.mark.parametrize("num", [1, 5, 17, 40, 90, 150])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_decode_step_follows_the_group_by_low_bits_only(num, temperature):
    """Every size of batch against single sequences: tokens differ at most where sums of another order may decide (hardly ever)."""
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=256, device=DEV)
    rng = wl.rng_for(5, num)
    lens = [int(x) for x in rng.integers(1, 120, num)]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    kv4 = sess.kv4_cache(blocks)
    sess.kv4_store(kv, kv4, bt, i32([0] * num), i32(lens), max(lens))
    ids = torch.arange(num, device=DEV)
    sampling = lambda ids: B.make_sampling(temperature, 77, ids.long()) if temperature else None
    for cache in (None, kv4):
        together = sess.decode_mx4(kv, bt, i32(lens), tok, cache, sampling=sampling(ids)).clone()
        alone = torch.cat([sess.decode_mx4(kv, bt[s:s + 1], i32(lens[s:s + 1]), tok[s:s + 1].contiguous(), cache,
                                           sampling=sampling(ids[s:s + 1])).clone() for s in range(num)])
        assert int((together != alone).sum()) <= max(1, num // 20)
    sess.close()


def test_decode_step_flags_sequences_of_a_table_of_its_own():
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=256, device=DEV)
    rng = wl.rng_for(5, 1)
    lens = [20, 33, 40, 15]
    table, blocks = wl.make_block_table(rng, [n + 1 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    table4, blocks4 = wl.make_block_table(wl.rng_for(6, 1), [n + 1 for n in lens], 16, max_blocks_per_seq=bt.shape[1] + 2)
    bt4, kv4 = torch.as_tensor(table4, device=DEV), sess.kv4_cache(blocks4)
    sess.kv4_store(kv, kv4, bt, i32([0] * 4), i32(lens), 40, kv4_block_table=bt4)
    mirror = sess.kv4_cache(blocks)
    sess.kv4_store(kv, mirror, bt, i32([0] * 4), i32(lens), 40)
    status = i32([9] * 4)
    want = sess.decode_mx4(kv, bt, i32(lens), tok, mirror, seq_status=status).clone()
    assert status.tolist() == [0] * 4
    got = sess.decode_mx4(kv, bt, i32(lens), tok, kv4, kv4_block_table=bt4, seq_status=status)
    assert status.tolist() == [0] * 4 and torch.equal(got, want)
    bt4[1, 2] = blocks4
    bt4[3, 2] = -1                                                # (not needed)
    bad_tok = tok.clone()
    bad_tok[2] = shape.vocab
    got = sess.decode_mx4(kv, bt, i32(lens), bad_tok, kv4, kv4_block_table=bt4, seq_status=status)
    assert status.tolist() == [0, B.LLM42_SEQ_BAD_BLOCK, B.LLM42_SEQ_BAD_TOKEN, 0]
    assert got.tolist() == [int(want[0]), -1, -1, int(want[3])]
    with pytest.raises(B.Llm42Error) as e:
        sess.decode_mx4(kv, bt, i32(lens), tok, kv4, kv4_block_table=bt4[:, :2].contiguous(), max_context=48)
    assert e.value.status == B.LLM42_ECAPACITY
    sess.close()


def test_decode_step_in_a_graph():
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=5), max_position=256, device=DEV)
    rng = wl.rng_for(5, 9)
    lens = [20, 33, 40]
    table, blocks = wl.make_block_table(rng, [n + 8 for n in lens], 16, spare_blocks=1)
    bt, kv = torch.as_tensor(table, device=DEV), sess.kv_cache(blocks)
    tok = sess.prefill(kv, bt, [wl.random_tokens(rng, n, shape.vocab) for n in lens], window=32)
    kv4 = sess.kv4_cache(blocks)
    sess.kv4_store(kv, kv4, bt, i32([0] * 3), i32(lens), 40)
    seq, cur, out = i32(lens), tok.clone(), torch.zeros_like(tok)
    want, s, c = [], seq.clone(), tok.clone()
    for _ in range(5):
        c = sess.decode_mx4(kv, bt, s, c, kv4).clone()
        s += 1
        want.append(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sess.decode_mx4(kv, bt, seq, cur, kv4, out_tokens=out)
        cur.copy_(out)
        seq += 1
    seq.copy_(i32(lens))
    cur.copy_(tok)
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cur, w)
    sess.close()


@pytest.mark.parametrize("fast", ["mx4", "mx4_cache"])
@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_the_loop_releases_the_verifiers_stream_whatever_the_fast_path_proposes(fast, temperature):
    shape = wl.TINY
    sess = VerifierSession(shape, wl.make_weights(shape, seed=42), max_position=512, device=DEV)
    rng = wl.rng_for(42, 4)
    lens = [9, 30, 64, 17, 48]
    prompts = [wl.random_tokens(rng, n, shape.vocab) for n in lens]
    sampling = B.make_sampling(temperature, 3) if temperature else None

    def state():
        table, blocks = wl.make_block_table(wl.rng_for(42, 6), [n + 80 for n in lens], 16, spare_blocks=2)
        kv, bt = sess.kv_cache(blocks), torch.as_tensor(table, device=DEV)
        return kv, bt, i32(lens), sess.prefill(kv, bt, prompts, window=16, sampling=sampling)

    kv, bt, seq, first = state()
    want = dvr.generate_verifier_only(sess, kv, bt, seq, first, 48, sampling=sampling)
    kv, bt, seq, first = state()
    got, stats = dvr.generate(sess, kv, bt, seq, first, 48, 8, sampling=sampling, fast=fast)
    assert torch.equal(got, want)
    assert stats.fast_tokens == stats.iterations * 5 * 7
    sess.close()


@pytest.mark.parametrize("fast", ["mx4", "mx4_cache"])
def test_the_statistics_command_runs_on_either_fast_path(fast, monkeypatch, capsys):
    monkeypatch.setattr(wl, "LLAMA_8B", wl.TINY)
    monkeypatch.setattr("sys.argv", ["dvr_stats", "--layers", "1", "--groups", "1,3", "--windows", "4", "--new", "6", "--prompt", "5,20", "--fast", fast])
    dvr_stats.main()                                             # (ends the process where a stream depended on its group)
    line = json.loads(capsys.readouterr().out.splitlines()[-1])
    assert line["fast"] == fast and line["all_streams_equal"] and len(line["rows"]) == 2
