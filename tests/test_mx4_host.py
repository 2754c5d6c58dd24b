"""The 4-bit operators' checks of host-visible arguments, and the reference that their GPU tests use, without a GPU."""
import ctypes

import pytest
import torch

import mx4_reference as ref
from paper_2601_17768_amd import binding as B

SZ = ctypes.c_size_t
KV = lambda base=4096, blocks=4, table=4096, width=4: B.KVCache(base, blocks, table, width)


def test_reference_rounds_to_the_nearest_level_and_ties_to_the_even_one():
    x = torch.zeros(32, dtype=torch.float64)
    x[:14] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.99, -0.25, -0.76, -3.49, 0.2499])
    assert ref.quantized(x)[:14].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -1, -3, 0]
    assert ref.quantized(2.0 ** -20 * x)[:14].tolist() == [2.0 ** -20 * v for v in [4, 0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -1, -3, 0]]
    assert bool(torch.isnan(ref.quantized(torch.tensor([1.0] * 31 + [float("inf")] + [2.0])))[:32].all())


def test_sizes_and_null_arguments_are_checked_without_a_gpu():
    lib, out = B.load_library(), SZ()
    assert lib.llm42_mx4_bytes(688, 256, ctypes.byref(out)) == B.LLM42_OK and out.value == 43 * 2176
    assert lib.llm42_mx4_bytes(1, 257, ctypes.byref(out)) == B.LLM42_OK and out.value == 2 * 2176
    for rows, cols in ((0, 4), (4, 0), (-1, 4), (2 ** 30 + 1, 4), (4, 2 ** 26 + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert lib.llm42_mx4_bytes(rows, cols, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_mx4_matmul_workspace_bytes(17, 5, 33, ctypes.byref(out)) == B.LLM42_OK and out.value == 32 * 64 * 2
    assert lib.llm42_mx4_matmul_workspace_bytes(B.LLM42_MAX_ROWS + 1, 5, 33, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_mx4_matmul_workspace_bytes(17, 5, 2 ** 26 + 1, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_kv4_bytes(None, 4, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_kv4_attention_workspace_bytes(None, 1, 1, 64, ctypes.byref(out)) == B.LLM42_EINVAL
    assert lib.llm42_decode_step_mx4_workspace_bytes(None, 1, 64, ctypes.byref(out)) == B.LLM42_EINVAL
    handle = ctypes.c_void_p()
    assert lib.llm42_mx4_model_create(None, ctypes.byref(handle)) == B.LLM42_EINVAL
    lib.llm42_mx4_model_destroy(None)


# (addresses that no kernel ever sees: every call here is refused)
QUANTIZE = dict(src=4096, type=B.LLM42_BF16, stride=64, rows=16, cols=64, dst=4096, dst_bytes=1 << 20, stream=None)
@pytest.mark.parametrize("bad,code", [
    (dict(src=None), B.LLM42_EINVAL), (dict(dst=None), B.LLM42_EINVAL), (dict(rows=0), B.LLM42_EINVAL), (dict(cols=-3), B.LLM42_EINVAL),
    (dict(type=7), B.LLM42_EINVAL), (dict(stride=63), B.LLM42_EINVAL), (dict(src=4097), B.LLM42_EINVAL),
    (dict(src=4098, type=B.LLM42_F32), B.LLM42_EINVAL), (dict(dst=4104), B.LLM42_EINVAL), (dict(dst_bytes=2175), B.LLM42_EWORKSPACE),
    (dict(rows=2 ** 30 + 1), B.LLM42_EINVAL), (dict(cols=2 ** 26 + 1, stride=2 ** 27), B.LLM42_EINVAL),
    (dict(rows=2 ** 31 - 1, cols=2 ** 31 - 1, stride=2 ** 31, dst_bytes=2 ** 63), B.LLM42_EINVAL)])
def test_quantize_and_dequantize_refuse(bad, code):
    lib, a = B.load_library(), {**QUANTIZE, **bad}
    assert lib.llm42_mx4_quantize(*a.values()) == code
    assert lib.llm42_mx4_dequantize(a["dst"], a["dst_bytes"], a["rows"], a["cols"], a["src"], a["type"], a["stride"], None) == code


MATMUL = dict(w=4096, w_bytes=1 << 20, n=16, k=64, x=4096, xs=64, rows=3, out=4096, type=B.LLM42_BF16, os=16, ws=None, ws_bytes=0, stream=None)
@pytest.mark.parametrize("bad,code", [
    (dict(w=None), B.LLM42_EINVAL), (dict(x=None), B.LLM42_EINVAL), (dict(out=None), B.LLM42_EINVAL), (dict(n=0), B.LLM42_EINVAL),
    (dict(k=0), B.LLM42_EINVAL), (dict(rows=0), B.LLM42_EINVAL), (dict(rows=B.LLM42_MAX_ROWS + 1), B.LLM42_EINVAL),
    (dict(xs=63), B.LLM42_EINVAL), (dict(os=15), B.LLM42_EINVAL), (dict(type=2), B.LLM42_EINVAL), (dict(x=4097), B.LLM42_EINVAL),
    (dict(w_bytes=2175), B.LLM42_EWORKSPACE), (dict(k=2 ** 26 + 1, xs=2 ** 27, w_bytes=2 ** 62), B.LLM42_EINVAL),
    # rows that are not 4-byte aligned, and more than 16 that are not 16-byte aligned or whose k is not a multiple of 32, need the workspace
    (dict(x=4098), B.LLM42_EWORKSPACE), (dict(xs=65), B.LLM42_EWORKSPACE), (dict(rows=17, x=4100), B.LLM42_EWORKSPACE), (dict(rows=17, xs=66), B.LLM42_EWORKSPACE), (dict(rows=17, k=63), B.LLM42_EWORKSPACE),
    (dict(rows=17, k=63, ws=4096, ws_bytes=2 * 32 * 64 - 1), B.LLM42_EWORKSPACE),
    (dict(rows=17, k=63, ws=4160, ws_bytes=1 << 20), B.LLM42_EWORKSPACE)])
def test_matmul_refuses(bad, code):
    assert B.load_library().llm42_mx4_matmul(*{**MATMUL, **bad}.values()) == code


def test_calls_of_a_model_refuse_null():
    lib, kv = B.load_library(), KV()
    assert lib.llm42_kv4_store(None, ctypes.byref(kv), ctypes.byref(kv), 4096, 4096, 1, 1, None, None) == B.LLM42_EINVAL
    assert lib.llm42_kv4_read(None, ctypes.byref(kv), 4096, 4096, 1, 1, 4096, 4096, None, None) == B.LLM42_EINVAL
    assert lib.llm42_kv4_attention(None, 0, ctypes.byref(kv), 4096, 64, 4096, 1, None, 1, 64, 4096, 64, None, 4096, 1 << 20, None) == B.LLM42_EINVAL
    assert lib.llm42_decode_step_mx4(None, ctypes.byref(kv), None, 4096, 4096, 1, 64, 4096, None, 4096, 1 << 30, None, None) == B.LLM42_EINVAL
    assert b"null" in lib.llm42_last_error()


def test_the_binding_refuses_tensors_that_are_not_on_the_device():
    with pytest.raises(ValueError):
        B.llm42_mx4_quantize(torch.zeros(4, 64), torch.zeros(2176, dtype=torch.uint8))
