"""ctypes binding of the verifier library (include/llm42.h, include/llm42_mx4.h, include/llm42_paged.h).

Argument marshalling only: every function here has the name and meaning of the
C entry point it wraps, takes torch tensors where the C call takes device
pointers, and raises `Llm42Error` on a negative status.  No step of the
verifier runs in Python; if libllm42.so is missing the import of the library
fails loudly - there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libllm42.so")

LLM42_OK, LLM42_EINVAL, LLM42_ESHAPE, LLM42_EWORKSPACE, LLM42_ECAPACITY, LLM42_EHIP = 0, -1, -2, -3, -4, -5
LLM42_KV_BLOCK = 16
LLM42_MAX_WINDOW = 512
LLM42_MAX_ROWS = 65536
LLM42_STATIC_SCRATCH_BYTES = 64 << 20
LLM42_BF16, LLM42_F32 = 0, 1
LLM42_ROPE_HALF, LLM42_ROPE_INTERLEAVED = 0, 1
LLM42_ROPE_NONE, LLM42_ROPE_LINEAR, LLM42_ROPE_LLAMA3, LLM42_ROPE_YARN = 0, 1, 2, 3
LLM42_MAX_SELECTED = 4096
LLM42_SEQ_OK, LLM42_SEQ_BAD_LENGTH, LLM42_SEQ_BAD_BLOCK, LLM42_SEQ_BAD_TOKEN = 0, 1, 2, 4

EXPORTS = ("llm42_model_create", "llm42_model_destroy", "llm42_kv_bytes", "llm42_workspace_bytes",
           "llm42_verify_window", "llm42_verify_window_static", "llm42_commit_rollback", "llm42_last_error", "llm42_schedule_info",
           "llm42_profile_enable", "llm42_profile_collect", "llm42_measure_verify_window_batch_chosen", "llm42_measure_attention_plan", "llm42_decode_step", "llm42_verify_window_sampled",
           "llm42_decode_step_sampled", "llm42_prefill", "llm42_prefill_workspace_bytes",
           "llm42_mx4_bytes", "llm42_mx4_quantize", "llm42_mx4_dequantize", "llm42_mx4_matmul_workspace_bytes", "llm42_mx4_matmul",
           "llm42_kv4_bytes", "llm42_kv4_store", "llm42_kv4_read", "llm42_kv4_attention_workspace_bytes", "llm42_kv4_attention",
           "llm42_mx4_model_create", "llm42_mx4_model_destroy", "llm42_decode_step_mx4_workspace_bytes", "llm42_decode_step_mx4",
           "llm42_heads_kv_bytes", "llm42_model_heads", "llm42_rope_create", "llm42_rope_destroy", "llm42_kv_append", "llm42_kv_bounds_bytes", "llm42_kv_bounds_store",
           "llm42_kv_bounds_read", "llm42_kv_select_workspace_bytes", "llm42_kv_select", "llm42_kv_sparse_attention_workspace_bytes",
           "llm42_kv_sparse_attention", "llm42_decode_step_sparse_workspace_bytes", "llm42_decode_step_sparse")
KERNEL_CLASSES = ("prepare", "embed", "rmsnorm", "qkv", "attention", "o_proj", "gate_up", "down", "lm_head",
                  "argmax", "commit")


class Llm42Error(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"llm42 status {status}: {message}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("kv_block_size", ctypes.c_int32), ("max_position", ctypes.c_int32)]


class Weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p), ("lm_head", ctypes.c_void_p)] + \
               [(n, ctypes.POINTER(ctypes.c_void_p)) for n in
                ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class Sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("seed", ctypes.c_uint64), ("request_ids", ctypes.c_void_p)]


def make_sampling(temperature: float, seed: int, request_ids: Optional[torch.Tensor] = None) -> Sampling:
    """request_ids: int64 device tensor [num_seqs] or None (then the index in the call is the id); the result keeps it."""
    sampling = Sampling(float(temperature), int(seed) & ((1 << 64) - 1), _ptr(request_ids, torch.int64))
    sampling.ids_tensor = request_ids                # (the struct holds a bare address)
    return sampling


class KVCache(ctypes.Structure):
    _fields_ = [("kv_base", ctypes.c_void_p), ("num_blocks", ctypes.c_int64), ("block_table", ctypes.c_void_p),
                ("max_blocks_per_seq", ctypes.c_int32)]


class Heads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim")]


class RopeConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rot_dim", "layout", "scaling", "max_position", "original_max_position")] + \
               [(n, ctypes.c_double) for n in ("theta", "factor", "low_freq_factor", "high_freq_factor", "beta_fast", "beta_slow",
                                               "attention_factor")]


_lib = None


def load_library(path: Optional[str] = None):
    """dlopen libllm42.so (built by paper_2601_17768_amd.build) and declare its signatures."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is not built; run `python -m paper_2601_17768_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.llm42_model_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(Weights), ctypes.POINTER(vp)]
    lib.llm42_model_create.restype = i32
    lib.llm42_model_destroy.argtypes = [vp]
    lib.llm42_model_destroy.restype = None
    lib.llm42_kv_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.llm42_kv_bytes.restype = i32
    lib.llm42_workspace_bytes.argtypes = [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.llm42_workspace_bytes.restype = i32
    lib.llm42_verify_window.argtypes = [vp, ctypes.POINTER(KVCache), vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, i32,
                                        vp, ctypes.c_size_t, vp]
    lib.llm42_verify_window.restype = i32
    lib.llm42_verify_window_static.argtypes = [vp, ctypes.POINTER(KVCache), vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, i32, vp]
    lib.llm42_verify_window_static.restype = i32
    lib.llm42_verify_window_sampled.argtypes = lib.llm42_verify_window.argtypes + [ctypes.POINTER(Sampling)]
    lib.llm42_verify_window_sampled.restype = i32
    lib.llm42_decode_step.argtypes = [vp, ctypes.POINTER(KVCache), vp, vp, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.llm42_decode_step.restype = i32
    lib.llm42_decode_step_sampled.argtypes = lib.llm42_decode_step.argtypes + [ctypes.POINTER(Sampling)]
    lib.llm42_decode_step_sampled.restype = i32
    lib.llm42_prefill_workspace_bytes.argtypes = lib.llm42_workspace_bytes.argtypes
    lib.llm42_prefill_workspace_bytes.restype = i32
    lib.llm42_prefill.argtypes = [vp, ctypes.POINTER(KVCache), vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, ctypes.c_size_t,
                                  vp, ctypes.POINTER(Sampling)]
    lib.llm42_prefill.restype = i32
    lib.llm42_commit_rollback.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    lib.llm42_commit_rollback.restype = i32
    lib.llm42_profile_enable.argtypes = [i32, i32]
    lib.llm42_profile_enable.restype = i32
    lib.llm42_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32), i32,
                                          ctypes.POINTER(i32)]
    lib.llm42_profile_collect.restype = i32
    lib.llm42_measure_verify_window_batch_chosen.argtypes = lib.llm42_verify_window.argtypes
    lib.llm42_measure_verify_window_batch_chosen.restype = i32
    lib.llm42_measure_attention_plan.argtypes = [vp, i32, i32, i32, ctypes.POINTER(i64)]
    lib.llm42_measure_attention_plan.restype = i32
    size, size_p, kvp = ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(KVCache)
    for name, args in {
            "llm42_mx4_bytes": [i32, i32, size_p],
            "llm42_mx4_quantize": [vp, i32, i64, i32, i32, vp, size, vp],
            "llm42_mx4_dequantize": [vp, size, i32, i32, vp, i32, i64, vp],
            "llm42_mx4_matmul_workspace_bytes": [i32, i32, i32, size_p],
            "llm42_mx4_matmul": [vp, size, i32, i32, vp, i64, i32, vp, i32, i64, vp, size, vp],
            "llm42_kv4_bytes": [vp, i64, size_p],
            "llm42_kv4_store": [vp, kvp, kvp, vp, vp, i32, i32, vp, vp],
            "llm42_kv4_read": [vp, kvp, vp, vp, i32, i32, vp, vp, vp, vp],
            "llm42_kv4_attention_workspace_bytes": [vp, i32, i32, i32, size_p],
            "llm42_kv4_attention": [vp, i32, kvp, vp, i64, vp, i32, vp, i32, i32, vp, i64, vp, vp, size, vp],
            "llm42_mx4_model_create": [vp, ctypes.POINTER(vp)],
            "llm42_decode_step_mx4_workspace_bytes": [vp, i32, i32, size_p],
            "llm42_decode_step_mx4": [vp, kvp, kvp, vp, vp, i32, i32, vp, vp, vp, size, vp, ctypes.POINTER(Sampling)]}.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i32
    hp, f32 = ctypes.POINTER(Heads), ctypes.c_float
    for name, args in {
            "llm42_heads_kv_bytes": [hp, i64, size_p],
            "llm42_model_heads": [vp, hp],
            "llm42_rope_create": [ctypes.POINTER(RopeConfig), ctypes.POINTER(vp)],
            "llm42_kv_append": [hp, i32, kvp, vp, vp, i64, vp, i64, vp, i64, i32, vp, vp, f32, vp, vp, i32, vp, i32, i32, vp, i64, vp, vp],
            "llm42_kv_bounds_bytes": [hp, i64, size_p],
            "llm42_kv_bounds_store": [hp, i32, kvp, vp, vp, vp, i32, i32, vp, vp],
            "llm42_kv_bounds_read": [hp, vp, i64, vp, i32, vp, vp, vp],
            "llm42_kv_select_workspace_bytes": [hp, i32, i32, i32, i32, size_p],
            "llm42_kv_select": [hp, i32, kvp, vp, vp, i64, vp, i32, vp, i32, i32, i32, i32, i32, vp, vp, vp, size, vp],
            "llm42_kv_sparse_attention_workspace_bytes": [hp, i32, i32, i32, size_p],
            "llm42_decode_step_sparse_workspace_bytes": [vp, i32, i32, i32, size_p],
            "llm42_decode_step_sparse": [vp, kvp, vp, i32, i32, i32, vp, vp, i32, i32, vp, vp, vp, size, vp, ctypes.POINTER(Sampling)],
            "llm42_kv_sparse_attention": [hp, i32, kvp, vp, i64, vp, i32, vp, i32, i32, vp, i32, f32, vp, i64, vp, vp, size, vp]}.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i32
    lib.llm42_rope_destroy.argtypes = [vp]
    lib.llm42_rope_destroy.restype = None
    lib.llm42_mx4_model_destroy.argtypes = [vp]
    lib.llm42_mx4_model_destroy.restype = None
    lib.llm42_last_error.argtypes = []
    lib.llm42_last_error.restype = ctypes.c_char_p
    lib.llm42_schedule_info.argtypes = []
    lib.llm42_schedule_info.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != LLM42_OK:
        raise Llm42Error(status, load_library().llm42_last_error().decode())


def _ptr(t: Optional[torch.Tensor], dtype: Optional[torch.dtype] = None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        # (the handle alone: without the Stream object around it 0.4 instead of 2.8 us a call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    return stream.cuda_stream or None


def _kv_view(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor, num_seqs: int) -> KVCache:
    """The C struct for a KV tensor and its block table; refuses a tensor smaller than num_blocks blocks need
    (the library sees a bare pointer and could not tell)."""
    if block_table.dim() != 2 or block_table.shape[0] != num_seqs:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq]")
    need = llm42_kv_bytes(model, num_blocks)
    if kv_base.numel() * kv_base.element_size() < need:
        raise ValueError(f"kv_base holds {kv_base.numel() * kv_base.element_size()} bytes, {num_blocks} blocks need {need}")
    return KVCache(_ptr(kv_base), num_blocks, _ptr(block_table, torch.int32), block_table.shape[1])


def make_config(shape, max_position: int) -> Config:
    """`shape` is any object with the model-dimension attributes (e.g. workloads.ModelShape)."""
    return Config(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                  shape.vocab, float(shape.rope_theta), float(shape.rms_eps), int(shape.kv_block_size),
                  int(max_position))


def llm42_model_create(cfg: Config, weights: Dict) -> int:
    """weights: {'embed','final_norm','lm_head': tensor, 'layers': [ {name: tensor} ]}, bf16 DEVICE
    tensors in [out_features, in_features] order.  Returns the opaque model handle."""
    lib = load_library()
    n = cfg.n_layers
    w = Weights()
    keep = []
    for name in ("embed", "final_norm", "lm_head"):
        setattr(w, name, _ptr(weights[name], torch.bfloat16))
    for name in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
        arr = (ctypes.c_void_p * n)(*[_ptr(weights["layers"][l][name], torch.bfloat16) for l in range(n)])
        keep.append(arr)
        setattr(w, name, ctypes.cast(arr, ctypes.POINTER(ctypes.c_void_p)))
    torch.cuda.synchronize()                       # the source tensors must be complete
    handle = ctypes.c_void_p()
    _check(lib.llm42_model_create(ctypes.byref(cfg), ctypes.byref(w), ctypes.byref(handle)))
    return handle.value


def llm42_model_destroy(model: int) -> None:
    load_library().llm42_model_destroy(model)


def llm42_kv_bytes(model: int, num_blocks: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_kv_bytes(model, num_blocks, ctypes.byref(out)))
    return out.value


def llm42_workspace_bytes(model: int, max_seqs: int, window: int, max_context: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_workspace_bytes(model, max_seqs, window, max_context, ctypes.byref(out)))
    return out.value


def llm42_verify_window(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor,
                        seq_lens: torch.Tensor, candidates: torch.Tensor, window: int,
                        n_valid: Optional[torch.Tensor], max_context: int, out_tokens: torch.Tensor,
                        workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None,
                        out_logits: Optional[torch.Tensor] = None, dump_seq_ids: Optional[torch.Tensor] = None,
                        stream=None, sampling: Optional[Sampling] = None, batch_chosen: bool = False) -> None:
    """sampling given: llm42_verify_window_sampled.  batch_chosen (measurement only):
    llm42_measure_verify_window_batch_chosen, the same pass off the fixed schedule."""
    num_seqs = seq_lens.numel()
    if candidates.shape != (num_seqs, window) or out_tokens.shape != (num_seqs, window):
        raise ValueError("candidates / out_tokens must be [num_seqs, window]")
    n_dump = 0 if dump_seq_ids is None else dump_seq_ids.numel()
    if n_dump and (out_logits is None or out_logits.shape[0] != n_dump or out_logits.shape[1] != window):
        raise ValueError("out_logits must be [n_dump, window, vocab]")
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    args = (model, ctypes.byref(kv), _ptr(seq_lens, torch.int32), _ptr(candidates, torch.int32), window,
            _ptr(n_valid, torch.int32), num_seqs, max_context, _ptr(out_tokens, torch.int32),
            _ptr(seq_status, torch.int32), _ptr(out_logits, torch.float32), _ptr(dump_seq_ids, torch.int32), n_dump,
            _ptr(workspace), workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if batch_chosen:
        if sampling is not None:
            raise ValueError("the measurement entry has no sampled form")
        _check(load_library().llm42_measure_verify_window_batch_chosen(*args))
    elif sampling is None:
        _check(load_library().llm42_verify_window(*args))
    else:
        _check(load_library().llm42_verify_window_sampled(*args, ctypes.byref(sampling)))


def llm42_verify_window_static(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor,
                               seq_lens: torch.Tensor, candidates: torch.Tensor, window: int,
                               n_valid: Optional[torch.Tensor], max_context: int, out_tokens: torch.Tensor,
                               seq_status: Optional[torch.Tensor] = None, out_logits: Optional[torch.Tensor] = None,
                               dump_seq_ids: Optional[torch.Tensor] = None, stream=None) -> None:
    """llm42_verify_window in the library's built-in scratch area (no workspace argument)."""
    num_seqs = seq_lens.numel()
    if candidates.shape != (num_seqs, window) or out_tokens.shape != (num_seqs, window):
        raise ValueError("candidates / out_tokens must be [num_seqs, window]")
    n_dump = 0 if dump_seq_ids is None else dump_seq_ids.numel()
    if n_dump and (out_logits is None or out_logits.shape[0] != n_dump or out_logits.shape[1] != window):
        raise ValueError("out_logits must be [n_dump, window, vocab]")
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_verify_window_static(
        model, ctypes.byref(kv), _ptr(seq_lens, torch.int32), _ptr(candidates, torch.int32), window,
        _ptr(n_valid, torch.int32), num_seqs, max_context, _ptr(out_tokens, torch.int32),
        _ptr(seq_status, torch.int32), _ptr(out_logits, torch.float32), _ptr(dump_seq_ids, torch.int32), n_dump,
        _stream_handle(stream)))


def llm42_decode_step(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor,
                      seq_lens: torch.Tensor, tokens: torch.Tensor, max_context: int, out_tokens: torch.Tensor,
                      workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None, stream=None,
                      sampling: Optional[Sampling] = None) -> None:
    """sampling given: llm42_decode_step_sampled."""
    num_seqs = seq_lens.numel()
    if tokens.numel() != num_seqs or out_tokens.numel() != num_seqs:
        raise ValueError("tokens / out_tokens must hold one entry per sequence")
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    args = (model, ctypes.byref(kv), _ptr(seq_lens, torch.int32), _ptr(tokens, torch.int32), num_seqs, max_context,
            _ptr(out_tokens, torch.int32), _ptr(seq_status, torch.int32), _ptr(workspace),
            workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if sampling is None:
        _check(load_library().llm42_decode_step(*args))
    else:
        _check(load_library().llm42_decode_step_sampled(*args, ctypes.byref(sampling)))


def llm42_prefill_workspace_bytes(model: int, max_seqs: int, chunk: int, max_context: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_prefill_workspace_bytes(model, max_seqs, chunk, max_context, ctypes.byref(out)))
    return out.value


def llm42_prefill(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor,
                  seq_lens: torch.Tensor, prompt_tokens: torch.Tensor, prompt_offsets: torch.Tensor,
                  max_prompt_len: int, chunk: int, max_context: int, out_next_tokens: torch.Tensor,
                  workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None, stream=None,
                  sampling: Optional[Sampling] = None) -> None:
    num_seqs = seq_lens.numel()
    if prompt_offsets.numel() != num_seqs + 1 or out_next_tokens.numel() != num_seqs:
        raise ValueError("prompt_offsets holds num_seqs + 1 entries, out_next_tokens one per sequence")
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_prefill(
        model, ctypes.byref(kv), _ptr(seq_lens, torch.int32), _ptr(prompt_tokens, torch.int32),
        _ptr(prompt_offsets, torch.int32), num_seqs, max_prompt_len, chunk, max_context,
        _ptr(out_next_tokens, torch.int32), _ptr(seq_status, torch.int32), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream),
        ctypes.byref(sampling) if sampling is not None else None))


_TYPES = {torch.bfloat16: LLM42_BF16, torch.float32: LLM42_F32}


def _on_current_device(*tensors: Optional[torch.Tensor]) -> None:
    """The library launches on the current device and sees bare pointers only."""
    at = {t.get_device() for t in tensors if t is not None}        # (-1: not on a GPU)
    if -1 in at or at != {torch._C._cuda_getDevice()}:
        raise ValueError("expected tensors on the current device")


def _matrix(t: torch.Tensor, rows: int, cols: int):
    """(pointer, type, row stride) of a plain matrix whose rows may lie apart."""
    if t.shape != (rows, cols):
        raise ValueError(f"expected a [{rows}, {cols}] tensor, got {tuple(t.shape)}")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"expected bfloat16 or float32, got {t.dtype}")
    apart, near = t.stride()
    if cols > 1 and near != 1:
        raise ValueError("the values of a row must be neighbours in memory")
    return t.data_ptr(), kind, apart if rows > 1 else cols


def _packed(t: torch.Tensor):
    if t.dtype != torch.uint8:
        raise ValueError(f"a 4-bit matrix is a uint8 tensor, got {t.dtype}")
    return _ptr(t), t.numel()


@functools.lru_cache(maxsize=1024)
def llm42_mx4_bytes(rows: int, cols: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_mx4_bytes(rows, cols, ctypes.byref(out)))
    return out.value


def llm42_mx4_quantize(src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
    """src [rows, cols], bfloat16 or float32; dst: uint8, llm42_mx4_bytes(rows, cols) or more."""
    if src.dim() != 2:
        raise ValueError("expected a matrix")
    _on_current_device(src, dst)
    rows, cols = src.shape
    p, kind, stride = _matrix(src, rows, cols)
    _check(load_library().llm42_mx4_quantize(p, kind, stride, rows, cols, *_packed(dst), _stream_handle(stream)))


def llm42_mx4_dequantize(src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
    """dst [rows, cols], bfloat16 or float32, receives what src stands for."""
    if dst.dim() != 2:
        raise ValueError("expected a matrix")
    _on_current_device(src, dst)
    rows, cols = dst.shape
    p, kind, stride = _matrix(dst, rows, cols)
    _check(load_library().llm42_mx4_dequantize(*_packed(src), rows, cols, p, kind, stride, _stream_handle(stream)))


def llm42_mx4_matmul_workspace_bytes(rows: int, n: int, k: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_mx4_matmul_workspace_bytes(rows, n, k, ctypes.byref(out)))
    return out.value


def llm42_mx4_matmul(w: torch.Tensor, x: torch.Tensor, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """out [rows, n] = x [rows, k] (bfloat16) times the transpose of the n x k matrix w."""
    if x.dim() != 2 or out.dim() != 2:
        raise ValueError("x and out must be matrices")
    _on_current_device(w, x, out, workspace)
    (rows, k), n = x.shape, out.shape[1]
    if x.dtype != torch.bfloat16:
        raise ValueError(f"x must be bfloat16, got {x.dtype}")
    xp, _, xs = _matrix(x, rows, k)
    op, kind, os_ = _matrix(out, rows, n)
    wp, wb = _packed(w)
    _check(load_library().llm42_mx4_matmul(wp, wb, n, k, xp, xs, rows, op, kind, os_, _ptr(workspace),
                                           0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_handle(stream)))


def llm42_kv4_bytes(model: int, num_blocks: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_kv4_bytes(model, num_blocks, ctypes.byref(out)))
    return out.value


def _kv4_view(model: int, kv4: torch.Tensor, num_blocks: int, block_table: torch.Tensor, num_seqs: int) -> KVCache:
    if block_table.dim() != 2 or block_table.shape[0] != num_seqs:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq]")
    need = llm42_kv4_bytes(model, num_blocks)
    if kv4.numel() * kv4.element_size() < need:
        raise ValueError(f"kv4 holds {kv4.numel() * kv4.element_size()} bytes, {num_blocks} blocks need {need}")
    return KVCache(_ptr(kv4), num_blocks, _ptr(block_table, torch.int32), block_table.shape[1])


def _per_seq(t: Optional[torch.Tensor], num_seqs: int):
    if t is not None and t.numel() != num_seqs:
        raise ValueError("expected one entry per sequence")
    return _ptr(t, torch.int32)


def llm42_kv4_store(model: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor, kv4_base: torch.Tensor,
                    kv4_num_blocks: int, kv4_block_table: torch.Tensor, first: torch.Tensor, count: torch.Tensor, max_count: int,
                    seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    num_seqs = first.numel()
    _on_current_device(kv_base, block_table, kv4_base, kv4_block_table, first, count, seq_status)
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    kv4 = _kv4_view(model, kv4_base, kv4_num_blocks, kv4_block_table, num_seqs)
    _check(load_library().llm42_kv4_store(model, ctypes.byref(kv), ctypes.byref(kv4), _per_seq(first, num_seqs), _per_seq(count, num_seqs),
                                          num_seqs, max_count, _per_seq(seq_status, num_seqs), _stream_handle(stream)))


def llm42_kv4_read(model: int, kv4_base: torch.Tensor, kv4_num_blocks: int, kv4_block_table: torch.Tensor, first: torch.Tensor,
                   count: torch.Tensor, max_count: int, out_k: torch.Tensor, out_v: torch.Tensor,
                   seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """out_k, out_v: bfloat16 [n_layers, num_seqs, max_count, n_kv_heads, head_dim]."""
    num_seqs = first.numel()
    _on_current_device(kv4_base, kv4_block_table, first, count, out_k, out_v, seq_status)
    kv4 = _kv4_view(model, kv4_base, kv4_num_blocks, kv4_block_table, num_seqs)
    if out_k.dim() != 5 or out_k.shape != out_v.shape or tuple(out_k.shape[1:3]) != (num_seqs, max_count):
        raise ValueError("out_k and out_v must be [n_layers, num_seqs, max_count, n_kv_heads, head_dim]")
    # a token's bytes in the cache are 17/32 of a byte a value: what kv4_bytes of one block says about layers, heads and head_dim
    layers, _, _, heads, hd = out_k.shape
    if llm42_kv4_bytes(model, 1) != layers * heads * hd * 17:
        raise ValueError("out_k and out_v do not have the model's layers, kv heads and head_dim")
    _check(load_library().llm42_kv4_read(model, ctypes.byref(kv4), _per_seq(first, num_seqs), _per_seq(count, num_seqs), num_seqs, max_count,
                                         _ptr(out_k, torch.bfloat16), _ptr(out_v, torch.bfloat16), _per_seq(seq_status, num_seqs),
                                         _stream_handle(stream)))


def llm42_kv4_attention_workspace_bytes(model: int, num_seqs: int, window: int, max_context: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_kv4_attention_workspace_bytes(model, num_seqs, window, max_context, ctypes.byref(out)))
    return out.value


def llm42_kv4_attention(model: int, layer: int, kv4_base: torch.Tensor, kv4_num_blocks: int, kv4_block_table: torch.Tensor,
                        q: torch.Tensor, seq_lens: torch.Tensor, n_valid: Optional[torch.Tensor], max_context: int, out: torch.Tensor,
                        workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """q, out: bfloat16 [num_seqs, window, n_q_heads, head_dim] with the model's heads; the rows of a token may lie apart, a token's heads may not."""
    num_seqs = seq_lens.numel()
    _on_current_device(kv4_base, kv4_block_table, q, seq_lens, n_valid, out, workspace, seq_status)
    if q.dim() != 4 or q.shape != out.shape or q.shape[0] != num_seqs:
        raise ValueError("q and out must be [num_seqs, window, n_q_heads, head_dim]")
    window, heads, hd = q.shape[1:]
    strides = []
    for t in (q, out):
        if t.dtype != torch.bfloat16:
            raise ValueError(f"expected bfloat16, got {t.dtype}")
        row = t.stride(1) if window > 1 else t.stride(0) if num_seqs > 1 else heads * hd
        if t.stride(3) != 1 or (heads > 1 and t.stride(2) != hd) or (num_seqs > 1 and window > 1 and t.stride(0) != window * row):
            raise ValueError("q and out: rows (sequence, token) at one distance from each other, their heads side by side")
        strides.append(row)
    kv4 = _kv4_view(model, kv4_base, kv4_num_blocks, kv4_block_table, num_seqs)
    _check(load_library().llm42_kv4_attention(model, layer, ctypes.byref(kv4), q.data_ptr(), strides[0], _per_seq(seq_lens, num_seqs), window,
                                              _per_seq(n_valid, num_seqs), num_seqs, max_context, out.data_ptr(), strides[1],
                                              _per_seq(seq_status, num_seqs), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                              _stream_handle(stream)))


def llm42_mx4_model_create(model: int) -> int:
    handle = ctypes.c_void_p()
    _check(load_library().llm42_mx4_model_create(model, ctypes.byref(handle)))
    return handle.value


def llm42_mx4_model_destroy(mx4: int) -> None:
    load_library().llm42_mx4_model_destroy(mx4)


def llm42_decode_step_mx4_workspace_bytes(mx4: int, max_seqs: int, max_context: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().llm42_decode_step_mx4_workspace_bytes(mx4, max_seqs, max_context, ctypes.byref(out)))
    return out.value


def llm42_decode_step_mx4(model: int, mx4: int, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor,
                          kv4_base: Optional[torch.Tensor], kv4_num_blocks: int, kv4_block_table: Optional[torch.Tensor],
                          seq_lens: torch.Tensor, tokens: torch.Tensor, max_context: int, out_tokens: torch.Tensor,
                          workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None, stream=None,
                          sampling: Optional[Sampling] = None) -> None:
    """kv4_base None: attention over the bf16 cache.  (`model`: the one that mx4 was made from, for the checks of the cache tensors.)"""
    num_seqs = seq_lens.numel()
    _on_current_device(kv_base, block_table, kv4_base, kv4_block_table, seq_lens, tokens, out_tokens, workspace, seq_status)
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    kv4 = None if kv4_base is None else _kv4_view(model, kv4_base, kv4_num_blocks, kv4_block_table, num_seqs)
    _check(load_library().llm42_decode_step_mx4(mx4, ctypes.byref(kv), None if kv4 is None else ctypes.byref(kv4), _per_seq(seq_lens, num_seqs),
                                                _per_seq(tokens, num_seqs), num_seqs, max_context, _per_seq(out_tokens, num_seqs),
                                                _per_seq(seq_status, num_seqs), _ptr(workspace),
                                                workspace.numel() * workspace.element_size(), _stream_handle(stream),
                                                ctypes.byref(sampling) if sampling is not None else None))


def _all_here(stream, *tensors: Optional[torch.Tensor]) -> Optional[int]:
    """_on_current_device and _stream_handle, at half the time."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError("expected tensors on the current device")
    return (torch._C._cuda_getCurrentRawStream(here) if stream is None else stream.cuda_stream) or None


def _dense(t: Optional[torch.Tensor], dtype: torch.dtype) -> Optional[int]:
    """Pointer of a tensor that has been found on the device."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


def _for_seqs(t: Optional[torch.Tensor], num_seqs: int) -> Optional[int]:
    if t is None:
        return None
    if t.numel() != num_seqs:
        raise ValueError("expected one entry per sequence")
    return _dense(t, torch.int32)


def _head_rows(t: torch.Tensor, shape):
    """(pointer, stride) of rows [num_seqs, window, heads, head_dim] at one distance from each other, their heads side by side."""
    if t.shape != shape:
        raise ValueError(f"expected {list(shape)}, got {list(t.shape)}")
    num_seqs, window, heads, head_dim = shape
    if t.is_contiguous():
        return t.data_ptr(), heads * head_dim
    of_seq, of_row, of_head, near = t.stride()
    row = of_row if window > 1 else of_seq if num_seqs > 1 else heads * head_dim
    if near != 1 or (heads > 1 and of_head != head_dim) or (num_seqs > 1 and window > 1 and of_seq != window * row):
        raise ValueError("rows (sequence, token) must lie at one distance from each other, their heads side by side")
    return t.data_ptr(), row


# (llm42_heads_kv_bytes and llm42_kv_bounds_bytes are reckoned by hand in what follows: a call of the library each would cost as much as all the rest)
def _paged_view(heads: Heads, kv: Optional[torch.Tensor], num_blocks: int, block_table: torch.Tensor, num_seqs: int) -> KVCache:
    shape = block_table.shape
    if len(shape) != 2 or shape[0] != num_seqs:
        raise ValueError("block_table must be [num_seqs, max_blocks_per_seq]")
    base = None
    if kv is not None:
        need = 64 * heads.n_layers * heads.n_kv_heads * heads.head_dim * num_blocks
        if kv.nbytes < need:
            raise ValueError(f"kv holds {kv.nbytes} bytes, {num_blocks} blocks need {need}")
        base = _dense(kv, kv.dtype)
    return KVCache(base, num_blocks, _dense(block_table, torch.int32), shape[1])


def _bounds(heads: Heads, bounds: torch.Tensor, num_blocks: int) -> int:
    need = heads.n_layers * heads.n_kv_heads * (2 * heads.head_dim + 16) * num_blocks
    if bounds.numel() < need:
        raise ValueError(f"bounds hold {bounds.numel()} bytes, {num_blocks} blocks need {need}")
    return _dense(bounds, torch.uint8)


def _workspace(t: Optional[torch.Tensor]):
    return (None, 0) if t is None else (_dense(t, t.dtype), t.nbytes)


def _lists(t: torch.Tensor, num_seqs: int, window: int, kv_heads: int) -> int:
    if t.dim() != 4 or t.shape[:3] != (num_seqs, window, kv_heads):
        raise ValueError(f"lists of blocks must be [{num_seqs}, {window}, {kv_heads}, entries], got {list(t.shape)}")
    return _dense(t, torch.int32)


def _asked(call, *args) -> int:
    out = ctypes.c_size_t()
    _check(call(*args, ctypes.byref(out)))
    return out.value


def llm42_heads_kv_bytes(heads: Heads, num_blocks: int) -> int:
    return _asked(load_library().llm42_heads_kv_bytes, ctypes.byref(heads), num_blocks)


def llm42_kv_bounds_bytes(heads: Heads, num_blocks: int) -> int:
    return _asked(load_library().llm42_kv_bounds_bytes, ctypes.byref(heads), num_blocks)


def llm42_model_heads(model: int) -> Heads:
    heads = Heads()
    _check(load_library().llm42_model_heads(model, ctypes.byref(heads)))
    return heads


def llm42_rope_create(cfg: RopeConfig) -> int:
    handle = ctypes.c_void_p()
    _check(load_library().llm42_rope_create(ctypes.byref(cfg), ctypes.byref(handle)))
    return handle.value


def llm42_rope_destroy(rope: int) -> None:
    load_library().llm42_rope_destroy(rope)


def llm42_kv_append(heads: Heads, layer: int, kv: torch.Tensor, num_blocks: int, block_table: torch.Tensor, bounds: Optional[torch.Tensor],
                    q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, q_norm: Optional[torch.Tensor], k_norm: Optional[torch.Tensor],
                    norm_eps: float, rope: Optional[int], seq_lens: torch.Tensor, n_valid: Optional[torch.Tensor], max_context: int,
                    q_out: Optional[torch.Tensor], seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """k, v [num_seqs, window, n_kv_heads, head_dim] and q [num_seqs, window, n_q_heads, head_dim]: bfloat16 or float32, all the same; q_out bfloat16.
    rope: a handle of llm42_rope_create."""
    num_seqs = seq_lens.numel()
    handle = _all_here(stream, kv, block_table, bounds, q, k, v, q_norm, k_norm, seq_lens, n_valid, q_out, seq_status)
    if k.dim() != 4:
        raise ValueError("k must be [num_seqs, window, n_kv_heads, head_dim]")
    window, hd, dtype = k.shape[1], heads.head_dim, k.dtype
    kind = _TYPES.get(dtype)
    if kind is None or v.dtype is not dtype or (q is not None and q.dtype is not dtype) or (q_out is not None and q_out.dtype is not torch.bfloat16):
        raise ValueError("q, k and v must be of one type, bfloat16 or float32, q_out bfloat16")
    of_kv, of_q = (num_seqs, window, heads.n_kv_heads, hd), (num_seqs, window, heads.n_q_heads, hd)
    kp, ks = _head_rows(k, of_kv)
    vp, vs = _head_rows(v, of_kv)
    qp, qs = (None, 0) if q is None else _head_rows(q, of_q)
    op, os_ = (None, 0) if q_out is None else _head_rows(q_out, of_q)
    for t in (q_norm, k_norm):
        if t is not None and t.numel() != hd:
            raise ValueError(f"gains hold {hd} values")
    view = _paged_view(heads, kv, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_kv_append(
        ctypes.byref(heads), layer, ctypes.byref(view), None if bounds is None else _bounds(heads, bounds, num_blocks), qp, qs, kp, ks, vp, vs, kind,
        _dense(q_norm, torch.bfloat16), _dense(k_norm, torch.bfloat16), norm_eps, rope, _for_seqs(seq_lens, num_seqs), window,
        _for_seqs(n_valid, num_seqs), num_seqs, max_context, op, os_, _for_seqs(seq_status, num_seqs), handle))


def llm42_kv_bounds_store(heads: Heads, layer: int, kv: torch.Tensor, num_blocks: int, block_table: torch.Tensor, bounds: torch.Tensor,
                          first: torch.Tensor, count: torch.Tensor, max_count: int, seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """layer -1: all."""
    num_seqs = first.numel()
    handle = _all_here(stream, kv, block_table, bounds, first, count, seq_status)
    view = _paged_view(heads, kv, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_kv_bounds_store(ctypes.byref(heads), layer, ctypes.byref(view), _bounds(heads, bounds, num_blocks),
                                                _for_seqs(first, num_seqs), _for_seqs(count, num_seqs), num_seqs, max_count,
                                                _for_seqs(seq_status, num_seqs), handle))


def llm42_kv_bounds_read(heads: Heads, bounds: torch.Tensor, num_blocks: int, block_ids: torch.Tensor, out_lo: torch.Tensor,
                         out_hi: torch.Tensor, stream=None) -> None:
    """out_lo, out_hi: bfloat16 [n_layers, len(block_ids), n_kv_heads, head_dim]."""
    handle = _all_here(stream, bounds, block_ids, out_lo, out_hi)
    shape = (heads.n_layers, block_ids.numel(), heads.n_kv_heads, heads.head_dim)
    if out_lo.shape != shape or out_hi.shape != shape:
        raise ValueError(f"out_lo and out_hi must be {list(shape)}")
    _check(load_library().llm42_kv_bounds_read(ctypes.byref(heads), _bounds(heads, bounds, num_blocks), num_blocks, _dense(block_ids, torch.int32),
                                               block_ids.numel(), _dense(out_lo, torch.bfloat16), _dense(out_hi, torch.bfloat16),
                                               handle))


def llm42_kv_select_workspace_bytes(heads: Heads, num_seqs: int, window: int, max_context: int, budget: int) -> int:
    return _asked(load_library().llm42_kv_select_workspace_bytes, ctypes.byref(heads), num_seqs, window, max_context, budget)


def llm42_kv_select(heads: Heads, layer: int, num_blocks: int, block_table: torch.Tensor, bounds: torch.Tensor, q: torch.Tensor,
                    seq_lens: torch.Tensor, n_valid: Optional[torch.Tensor], max_context: int, sink: int, recent: int, selected: torch.Tensor,
                    workspace: Optional[torch.Tensor], seq_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """selected: int32 [num_seqs, window, n_kv_heads, budget]."""
    num_seqs = seq_lens.numel()
    handle = _all_here(stream, block_table, bounds, q, seq_lens, n_valid, selected, workspace, seq_status)
    if q.dim() != 4 or q.dtype != torch.bfloat16:
        raise ValueError("q must be bfloat16 [num_seqs, window, n_q_heads, head_dim]")
    window = q.shape[1]
    shape = (num_seqs, window, heads.n_q_heads, heads.head_dim)
    qp, qs = _head_rows(q, shape)
    view = _paged_view(heads, None, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_kv_select(
        ctypes.byref(heads), layer, ctypes.byref(view), _bounds(heads, bounds, num_blocks), qp, qs, _for_seqs(seq_lens, num_seqs), window,
        _for_seqs(n_valid, num_seqs), num_seqs, max_context, selected.shape[-1], sink, recent,
        _lists(selected, num_seqs, window, heads.n_kv_heads), _for_seqs(seq_status, num_seqs), *_workspace(workspace), handle))


def llm42_kv_sparse_attention_workspace_bytes(heads: Heads, num_seqs: int, window: int, width: int) -> int:
    return _asked(load_library().llm42_kv_sparse_attention_workspace_bytes, ctypes.byref(heads), num_seqs, window, width)


def llm42_kv_sparse_attention(heads: Heads, layer: int, kv: torch.Tensor, num_blocks: int, block_table: torch.Tensor, q: torch.Tensor,
                              seq_lens: torch.Tensor, n_valid: Optional[torch.Tensor], max_context: int, selected: torch.Tensor, scale: float,
                              out: torch.Tensor, workspace: Optional[torch.Tensor], seq_status: Optional[torch.Tensor] = None,
                              stream=None) -> None:
    """q, out: bfloat16 [num_seqs, window, n_q_heads, head_dim]; selected: int32 [num_seqs, window, n_kv_heads, width]; scale 0: 1 / sqrt(head_dim)."""
    num_seqs = seq_lens.numel()
    handle = _all_here(stream, kv, block_table, q, seq_lens, n_valid, selected, out, workspace, seq_status)
    if q.dim() != 4 or q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16:
        raise ValueError("q and out must be bfloat16 [num_seqs, window, n_q_heads, head_dim]")
    window = q.shape[1]
    shape = (num_seqs, window, heads.n_q_heads, heads.head_dim)
    qp, qs = _head_rows(q, shape)
    op, os_ = _head_rows(out, shape)
    view = _paged_view(heads, kv, num_blocks, block_table, num_seqs)
    _check(load_library().llm42_kv_sparse_attention(
        ctypes.byref(heads), layer, ctypes.byref(view), qp, qs, _for_seqs(seq_lens, num_seqs), window, _for_seqs(n_valid, num_seqs), num_seqs,
        max_context, _lists(selected, num_seqs, window, heads.n_kv_heads), selected.shape[-1], scale, op, os_, _for_seqs(seq_status, num_seqs),
        *_workspace(workspace), handle))


def llm42_decode_step_sparse_workspace_bytes(model: int, max_seqs: int, max_context: int, budget: int) -> int:
    return _asked(load_library().llm42_decode_step_sparse_workspace_bytes, model, max_seqs, max_context, budget)


def llm42_decode_step_sparse(model: int, heads: Heads, kv_base: torch.Tensor, num_blocks: int, block_table: torch.Tensor, bounds: torch.Tensor,
                             budget: int, sink: int, recent: int, seq_lens: torch.Tensor, tokens: torch.Tensor, max_context: int,
                             out_tokens: torch.Tensor, workspace: torch.Tensor, seq_status: Optional[torch.Tensor] = None, stream=None,
                             sampling: Optional[Sampling] = None) -> None:
    """(`heads`: what the bounds were made with, which has to be the model's.)"""
    num_seqs = seq_lens.numel()
    handle = _all_here(stream, kv_base, block_table, bounds, seq_lens, tokens, out_tokens, workspace, seq_status)
    kv = _kv_view(model, kv_base, num_blocks, block_table, num_seqs)
    if bytes(llm42_model_heads(model)) != bytes(heads):
        raise ValueError("heads are not the model's")
    _check(load_library().llm42_decode_step_sparse(
        model, ctypes.byref(kv), _bounds(heads, bounds, num_blocks), budget, sink, recent, _for_seqs(seq_lens, num_seqs),
        _for_seqs(tokens, num_seqs), num_seqs, max_context, _for_seqs(out_tokens, num_seqs), _for_seqs(seq_status, num_seqs), *_workspace(workspace),
        handle, ctypes.byref(sampling) if sampling is not None else None))


def llm42_commit_rollback(candidates: torch.Tensor, out_tokens: torch.Tensor, n_valid: Optional[torch.Tensor],
                          seq_lens: torch.Tensor, committed_counts: torch.Tensor, committed_tokens: torch.Tensor,
                          rolled_back_counts: Optional[torch.Tensor] = None, stream=None) -> None:
    num_seqs, window = candidates.shape
    _check(load_library().llm42_commit_rollback(
        _ptr(candidates, torch.int32), _ptr(out_tokens, torch.int32), _ptr(n_valid, torch.int32), num_seqs, window,
        _ptr(seq_lens, torch.int32), _ptr(committed_counts, torch.int32), _ptr(committed_tokens, torch.int32),
        _ptr(rolled_back_counts, torch.int32), _stream_handle(stream)))


def llm42_schedule_info() -> str:
    return load_library().llm42_schedule_info().decode()


def llm42_measure_attention_plan(model: int, num_seqs: int, window: int, max_context: int) -> Dict:
    """How a call of this shape distributes its attention work (see llm42_measure.h)."""
    out = (ctypes.c_int64 * 5)()
    _check(load_library().llm42_measure_attention_plan(model, num_seqs, window, max_context, out))
    return {"item_keys": out[0], "direct": bool(out[1]), "may_take_sequences": bool(out[2]),
            "sequences_flag_offset": out[3], "streaming": out[4] == 1, "split": out[4] == 2, "waves": out[4] == 3, "may_take_waves": out[4] == 4}


def llm42_profile_enable(kind, max_launches: int) -> None:
    """kind: a name from KERNEL_CLASSES, or None for every class."""
    k = -1 if kind is None else KERNEL_CLASSES.index(kind)
    _check(load_library().llm42_profile_enable(k, max_launches))


def llm42_profile_collect(capacity: int):
    """Returns [(class name, milliseconds)] in launch order and disables timing."""
    ms = (ctypes.c_float * capacity)()
    kinds = (ctypes.c_int32 * capacity)()
    n = ctypes.c_int32()
    _check(load_library().llm42_profile_collect(ms, kinds, capacity, ctypes.byref(n)))
    return [(KERNEL_CLASSES[kinds[i]], float(ms[i])) for i in range(n.value)]
