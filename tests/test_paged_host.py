"""The checks of host-visible arguments of the operators around the paged cache, and the reference that their GPU tests use, without a GPU."""
import ctypes
import math

import pytest
import torch

import paged_reference as ref
from paper_2601_17768_amd import binding as B

SZ = ctypes.c_size_t
HEADS = lambda **kw: B.Heads(**{**dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128), **kw})
KV = lambda base=4096, blocks=4, table=4096, width=4: B.KVCache(base, blocks, table, width)


def test_reference_bounds_and_scores():
    k = torch.zeros(16, 4)
    k[3] = torch.tensor([127.0, -1.0, 0.5, 0.0])
    lo, hi = ref.bounds(k)
    assert lo.tolist() == [0, -1, 0, 0] and hi.tolist() == [127, 0, 1, 0]
    k[5, 0] = 128.0                                              # (the next power of two)
    lo, hi = ref.bounds(k)
    assert lo.tolist() == [0, -2, 0, 0] and hi.tolist() == [128, 0, 2, 0]
    assert ref.exponent(0.0) == -40 and ref.exponent(127 * 2.0 ** -40) == -40 and ref.exponent(128 * 2.0 ** -40) == -39
    k[0, 1] = math.nan
    assert math.isinf(ref.bounds(k)[1][0])
    q = torch.tensor([[1.0, -1.0, 0.0, 0.0]])
    lo, hi = torch.zeros(6, 4).double(), torch.zeros(6, 4).double()
    hi[2, 0], lo[3, 1], hi[4, 1] = 3.0, -3.0, 9.0                # scores 0 0 3 3 0 0
    assert ref.select(q, lo, hi, 5, 3, 0, 1) == [2, 3, 5] and ref.select(q, lo, hi, 5, 2, 0, 1) == [2, 5]
    assert ref.select(q, lo, hi, 5, 4, 1, 1) == [0, 2, 3, 5] and ref.select(q, lo, hi, 1, 4, 1, 1) == [0, 1, -1, -1]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_reference_rotation_keeps_products_of_distances(layout):
    q, k = torch.randn(64).double(), torch.randn(64).double()
    rope = (64, 1e4, layout, {"kind": "none"})
    at = lambda p, d: float(ref.turned(q, p + d, None, 0, rope) @ ref.turned(k, p, None, 0, rope))
    assert at(3, 5) == pytest.approx(at(40, 5), abs=1e-9) and at(3, 5) != pytest.approx(at(3, 6), abs=1e-3)


def test_sizes():
    lib, out = B.load_library(), SZ()
    h = HEADS()
    assert lib.llm42_heads_kv_bytes(ctypes.byref(h), 5, ctypes.byref(out)) == B.LLM42_OK and out.value == 2 * 2 * 5 * 2 * 16 * 128 * 2
    assert lib.llm42_kv_bounds_bytes(ctypes.byref(h), 5, ctypes.byref(out)) == B.LLM42_OK and out.value == 2 * 5 * 2 * 272
    assert lib.llm42_kv_bounds_bytes(ctypes.byref(h), -1, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_kv_bounds_bytes(ctypes.byref(h), 5, None) == B.LLM42_EINVAL
    assert lib.llm42_heads_kv_bytes(None, 5, ctypes.byref(out)) == B.LLM42_EINVAL
    for bad, code in ((dict(head_dim=96), B.LLM42_ESHAPE), (dict(n_kv_heads=3), B.LLM42_ESHAPE), (dict(n_q_heads=34), B.LLM42_ESHAPE),
                      (dict(n_layers=0), B.LLM42_EINVAL), (dict(n_kv_heads=0), B.LLM42_EINVAL), (dict(n_q_heads=2048, n_kv_heads=128), B.LLM42_EINVAL)):
        assert lib.llm42_kv_bounds_bytes(ctypes.byref(HEADS(**bad)), 5, ctypes.byref(out)) == code, bad
    for args in ((0, 1, 64, 8), (1, 0, 64, 8), (1, 513, 64, 8), (65537, 1, 64, 8), (1, 1, 0, 8), (1, 1, 2 ** 30 + 1, 8), (1, 1, 64, 0), (1, 1, 64, 4097)):
        assert lib.llm42_kv_select_workspace_bytes(ctypes.byref(h), *args, ctypes.byref(out)) == B.LLM42_EINVAL, args
    for args in ((0, 1, 8), (1, 513, 8), (1, 1, 0), (1, 1, 4097)):
        assert lib.llm42_kv_sparse_attention_workspace_bytes(ctypes.byref(h), *args, ctypes.byref(out)) == B.LLM42_EINVAL, args


ROPE = dict(rot_dim=64, layout=0, scaling=0, max_position=128, original_max_position=64, theta=1e4, factor=2.0, low_freq_factor=1.0,
            high_freq_factor=4.0, beta_fast=32.0, beta_slow=1.0, attention_factor=0.0)
@pytest.mark.parametrize("bad", [
    dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=130), dict(layout=2), dict(scaling=4), dict(scaling=-1), dict(max_position=0),
    dict(max_position=2 ** 24 + 1), dict(theta=1.0), dict(theta=math.nan), dict(theta=math.inf), dict(attention_factor=-1.0),
    dict(attention_factor=math.nan), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.inf), dict(scaling=2, original_max_position=0),
    dict(scaling=2, low_freq_factor=4.0), dict(scaling=2, low_freq_factor=0.0), dict(scaling=3, beta_slow=0.0), dict(scaling=3, beta_fast=0.5),
    dict(scaling=3, factor=math.nan)])
def test_rope_refuses(bad):
    handle = ctypes.c_void_p(1)
    cfg = B.RopeConfig(**{**ROPE, **bad})
    assert B.load_library().llm42_rope_create(ctypes.byref(cfg), ctypes.byref(handle)) == B.LLM42_EINVAL and handle.value is None
    assert B.load_library().llm42_rope_create(None, ctypes.byref(handle)) == B.LLM42_EINVAL


def call(name, args):
    return getattr(B.load_library(), name)(*(ctypes.byref(v) if isinstance(v, ctypes.Structure) else v for v in args.values()))


# (addresses that no kernel ever sees: every call here is refused)
APPEND = dict(heads=HEADS(), layer=1, kv=KV(), bounds=4096, q=4096, qs=1024, k=4096, ks=256, v=4096, vs=256, type=0, qn=None, kn=None, eps=1e-6,
              rope=None, lens=4096, window=2, valid=None, seqs=3, ctx=64, out=8192, os=1024, status=None, stream=None)
@pytest.mark.parametrize("bad,code", [
    (dict(heads=None), -1), (dict(heads=HEADS(head_dim=32)), -2), (dict(layer=2), -1), (dict(layer=-1), -1), (dict(kv=None), -1), (dict(kv=KV(base=None)), -1),
    (dict(kv=KV(base=4104)), -1), (dict(kv=KV(blocks=0)), -1), (dict(kv=KV(blocks=2 ** 31)), -1), (dict(kv=KV(table=None)), -1), (dict(kv=KV(width=0)), -1),
    (dict(bounds=4104), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(q=4104), -1), (dict(qs=1023), -1), (dict(qs=1016), -1), (dict(qs=1028), -1),
    (dict(k=None), -1), (dict(k=4098), -1), (dict(ks=255), -1), (dict(ks=252), -1), (dict(v=None), -1), (dict(vs=248), -1), (dict(type=2), -1),
    (dict(qn=4104), -1), (dict(kn=4097), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(lens=None), -1), (dict(window=0), -1),
    (dict(window=513), -1), (dict(seqs=0), -1), (dict(seqs=65536, window=2), -1), (dict(ctx=0), -1), (dict(ctx=65), -4), (dict(ctx=2 ** 30 + 1), -1),
    (dict(os=1020), -1), (dict(os=1028), -1), (dict(out=8200), -1),
    (dict(heads=HEADS(n_q_heads=1024, n_kv_heads=1024), seqs=65536, window=1, qs=1 << 17, os=1 << 17, ks=1 << 17, vs=1 << 17), -1)])
def test_append_refuses(bad, code):
    assert call("llm42_kv_append", {**APPEND, **bad}) == code


BOUNDS = dict(heads=HEADS(), layer=-1, kv=KV(), bounds=4096, first=4096, count=4096, seqs=3, most=64, status=None, stream=None)
@pytest.mark.parametrize("bad,code", [
    (dict(heads=None), -1), (dict(layer=-2), -1), (dict(layer=2), -1), (dict(kv=None), -1), (dict(kv=KV(base=None)), -1), (dict(bounds=None), -1),
    (dict(bounds=4100), -1), (dict(first=None), -1), (dict(count=None), -1), (dict(seqs=0), -1), (dict(most=0), -1),
    (dict(seqs=2 ** 25 + 1, most=1), -1), (dict(seqs=2 ** 20, most=2 ** 20), -1)])
def test_bounds_store_refuses(bad, code):
    assert call("llm42_kv_bounds_store", {**BOUNDS, **bad}) == code


def test_bounds_read_refuses():
    good = dict(heads=HEADS(), bounds=4096, blocks=4, ids=4096, n=2, lo=4096, hi=4096, stream=None)
    for bad in (dict(heads=None), dict(bounds=None), dict(bounds=4104), dict(blocks=0), dict(ids=None), dict(n=-1), dict(n=2 ** 26 + 1), dict(lo=None),
                dict(hi=4100)):
        assert call("llm42_kv_bounds_read", {**good, **bad}) == B.LLM42_EINVAL, bad
    assert call("llm42_kv_bounds_read", {**good, "n": 0}) == B.LLM42_OK


SELECT = dict(heads=HEADS(), layer=0, kv=KV(base=None), bounds=4096, q=4096, qs=1024, lens=4096, window=2, valid=None, seqs=3, ctx=64, budget=8, sink=1,
              recent=2, selected=4096, status=None, ws=None, ws_bytes=0, stream=None)
LONG = dict(kv=KV(base=None, width=2 ** 20), ctx=2 ** 23)
@pytest.mark.parametrize("bad,code", [
    (dict(heads=None), -1), (dict(layer=2), -1), (dict(kv=None), -1), (dict(kv=KV(blocks=0)), -1), (dict(bounds=None), -1), (dict(bounds=4104), -1),
    (dict(q=None), -1), (dict(q=4104), -1), (dict(qs=1020), -1), (dict(lens=None), -1), (dict(window=0), -1), (dict(seqs=0), -1), (dict(ctx=65), -4),
    (dict(budget=0), -1), (dict(budget=4097), -1), (dict(sink=-1), -1), (dict(recent=0), -1), (dict(sink=7), -1), (dict(sink=2 ** 31 - 1), -1),
    (dict(selected=None), -1), (dict(**LONG), -3), (dict(**LONG, ws=4096, ws_bytes=64), -3), (dict(**LONG, ws=4100, ws_bytes=2 ** 40), -3)])
def test_select_refuses(bad, code):
    assert call("llm42_kv_select", {**SELECT, **bad}) == code


ATTEND = dict(heads=HEADS(), layer=0, kv=KV(), q=4096, qs=1024, lens=4096, window=2, valid=None, seqs=3, ctx=64, selected=4096, width=8, scale=0.0,
              out=8192, os=1024, status=None, ws=None, ws_bytes=0, stream=None)
@pytest.mark.parametrize("bad,code", [
    (dict(heads=None), -1), (dict(layer=2), -1), (dict(kv=None), -1), (dict(kv=KV(base=None)), -1), (dict(q=None), -1), (dict(q=4104), -1),
    (dict(qs=1020), -1), (dict(lens=None), -1), (dict(window=513), -1), (dict(ctx=65), -4), (dict(selected=None), -1), (dict(width=0), -1),
    (dict(width=4097), -1), (dict(scale=-1.0), -1), (dict(scale=math.inf), -1), (dict(scale=math.nan), -1), (dict(out=None), -1), (dict(os=1020), -1),
    (dict(width=4096), -3), (dict(width=4096, ws=4096, ws_bytes=256), -3), (dict(width=4096, ws=4100, ws_bytes=2 ** 40), -3)])
def test_sparse_attention_refuses(bad, code):
    assert call("llm42_kv_sparse_attention", {**ATTEND, **bad}) == code


def test_sparse_step_refuses_without_a_model():
    lib, out = B.load_library(), SZ()
    assert lib.llm42_decode_step_sparse_workspace_bytes(None, 1, 64, 8, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_decode_step_sparse(None, None, None, 8, 1, 2, None, None, 1, 64, None, None, None, 0, None, None) == B.LLM42_EINVAL


@pytest.mark.parametrize("layers,kv_heads,hd", [(1, 1, 64), (3, 8, 128), (32, 5, 64)])
def test_the_bindings_sizes_are_the_librarys(layers, kv_heads, hd):
    """The binding checks buffers by its own arithmetic: one byte less than the library asks for is refused."""
    heads, blocks = B.Heads(layers, 2 * kv_heads, kv_heads, hd), 7
    table = torch.zeros((2, 3), dtype=torch.int32)
    kv, bounds = (torch.zeros(n(heads, blocks) - 1, dtype=torch.uint8) for n in (B.llm42_heads_kv_bytes, B.llm42_kv_bounds_bytes))
    for call in (lambda: B._paged_view(heads, kv, blocks, table, 2), lambda: B._bounds(heads, bounds, blocks)):
        with pytest.raises(ValueError, match="blocks need"):
            call()
    B._paged_view(heads, torch.zeros(len(kv) + 1, dtype=torch.uint8), blocks, table, 2)
    B._bounds(heads, torch.zeros(len(bounds) + 1, dtype=torch.uint8), blocks)
