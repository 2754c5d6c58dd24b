"""Buffer management around the binding: uploads weights, owns the model handle,
the workspace and the output tensors, and forwards to the two hot entry points.
No arithmetic of the verifier happens here."""
from __future__ import annotations

from typing import Dict, Optional, Sequence

import numpy as np
import torch

from . import binding as B


def _to_device(weights: Dict, device) -> Dict:
    out = {k: weights[k].to(device) for k in ("embed", "final_norm", "lm_head")}
    out["layers"] = [{k: v.to(device) for k, v in lw.items()} for lw in weights["layers"]]
    return out


class VerifierSession:
    """A model on one device and the workspace that its calls share: eager calls follow each other, whatever their streams."""

    def __init__(self, shape, weights: Dict, max_position: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("the verifier needs a GPU; there is no CPU path")
        self.shape = shape
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.cfg = B.make_config(shape, max_position)
        dev_w = weights if weights["embed"].is_cuda else _to_device(weights, self.device)
        self.model = B.llm42_model_create(self.cfg, dev_w)
        del dev_w
        self._mx4 = None
        self._attention4_need, self._decode4_need, self._decode_sparse_need = {}, {}, {}
        self._ws = None
        self._ws_key = None
        self._ws_captured, self._ws_kept = False, []
        self._index = torch.cuda.current_device()
        self._ws_stream, self._ws_handle = None, None            # the last call's, and its handle

    def close(self):
        if self.model:
            torch.cuda.synchronize()
            if self._mx4:
                B.llm42_mx4_model_destroy(self._mx4)
                self._mx4 = None
            B.llm42_model_destroy(self.model)
            self.model = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_cache(self, num_blocks: int, fill: float = 0.0) -> torch.Tensor:
        from .kv_layout import alloc_kv
        kv = alloc_kv(self.shape, num_blocks, self.device, fill)
        assert kv.numel() * 2 == B.llm42_kv_bytes(self.model, num_blocks)
        return kv

    def workspace(self, num_seqs: int, window: int, max_context: int) -> torch.Tensor:
        return self._room(B.llm42_workspace_bytes(self.model, num_seqs, window, max_context))

    def _room(self, need: int) -> torch.Tensor:
        """The session's workspace, of `need` bytes or more.  One that a captured call uses is kept when it is outgrown: the graph still writes it.
        Calls share it, so one on another stream than the last waits for that, and an outgrown one is free behind the work of every
        stream that used it.  (What a graph does when it is replayed is not seen here: replays are ordered by their caller.)"""
        capturing = torch.cuda.is_current_stream_capturing()
        if self._ws is None or self._ws.numel() < need:
            if self._ws_captured:
                self._ws_kept.append(self._ws)
            self._ws, self._ws_captured = torch.empty(need, dtype=torch.uint8, device=self.device), False
        self._ws_captured |= capturing
        handle = torch._C._cuda_getCurrentRawStream(self._index)
        if handle != self._ws_handle and not capturing:
            stream = torch.cuda.current_stream(self._index)
            if self._ws_stream is not None:
                stream.wait_stream(self._ws_stream)
            if not self._ws_captured:
                self._ws.record_stream(stream)
            self._ws_stream, self._ws_handle = stream, handle
        return self._ws

    def verify(self, kv: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
               candidates: torch.Tensor, n_valid: Optional[torch.Tensor] = None,
               dump_seq_ids: Optional[torch.Tensor] = None, max_context: Optional[int] = None,
               out_tokens: Optional[torch.Tensor] = None, out_logits: Optional[torch.Tensor] = None,
               seq_status: Optional[torch.Tensor] = None, sampling=None):
        """One llm42_verify_window call (llm42_verify_window_sampled if `sampling`, a binding.Sampling,
        is given).  Returns (out_tokens, seq_status, out_logits)."""
        num_seqs, window = candidates.shape
        if max_context is None:
            max_context = block_table.shape[1] * B.LLM42_KV_BLOCK
        ws = self.workspace(num_seqs, window, max_context)
        if out_tokens is None:
            out_tokens = torch.empty((num_seqs, window), dtype=torch.int32, device=self.device)
        if seq_status is None:
            seq_status = torch.empty(num_seqs, dtype=torch.int32, device=self.device)
        if dump_seq_ids is not None and out_logits is None:
            out_logits = torch.zeros((dump_seq_ids.numel(), window, self.shape.vocab), dtype=torch.float32,
                                     device=self.device)
        B.llm42_verify_window(self.model, kv, kv.shape[2], block_table, seq_lens, candidates, window, n_valid,
                              max_context, out_tokens, ws, seq_status, out_logits, dump_seq_ids, sampling=sampling)
        return out_tokens, seq_status, out_logits

    # ---- the fast path in 4 bits ----
    @property
    def mx4(self) -> int:
        """Handle of the model's 4-bit copy, made when it is first asked for (which no graph can hold: ask before a capture)."""
        if not self._mx4:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("the 4-bit copy of the model must be made before a capture")
            self._mx4 = B.llm42_mx4_model_create(self.model)
        return self._mx4

    def kv4_cache(self, num_blocks: int) -> torch.Tensor:
        """A 4-bit cache of num_blocks blocks."""
        shape = (self.shape.n_layers, num_blocks, self.shape.n_kv_heads, 17 * self.shape.head_dim)
        assert np.prod(shape) == B.llm42_kv4_bytes(self.model, num_blocks)
        return torch.empty(shape, dtype=torch.uint8, device=self.device)

    def kv4_store(self, kv: torch.Tensor, kv4: torch.Tensor, block_table: torch.Tensor, first: torch.Tensor, count: torch.Tensor,
                  max_count: int, kv4_block_table: Optional[torch.Tensor] = None, seq_status: Optional[torch.Tensor] = None) -> None:
        """One llm42_kv4_store call (the 4-bit cache has the bf16 cache's block table unless another is given)."""
        B.llm42_kv4_store(self.model, kv, kv.shape[2], block_table, kv4, kv4.shape[1],
                          block_table if kv4_block_table is None else kv4_block_table, first, count, max_count, seq_status)

    def kv4_read(self, kv4: torch.Tensor, block_table: torch.Tensor, first: torch.Tensor, count: torch.Tensor, max_count: int,
                 out_k: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None, seq_status: Optional[torch.Tensor] = None):
        """One llm42_kv4_read call.  Returns (out_k, out_v)."""
        shape = (self.shape.n_layers, first.numel(), max_count, self.shape.n_kv_heads, self.shape.head_dim)
        if out_k is None:
            out_k = torch.zeros(shape, dtype=torch.bfloat16, device=self.device)
        if out_v is None:
            out_v = torch.zeros(shape, dtype=torch.bfloat16, device=self.device)
        B.llm42_kv4_read(self.model, kv4, kv4.shape[1], block_table, first, count, max_count, out_k, out_v, seq_status)
        return out_k, out_v

    def kv4_attention(self, layer: int, kv4: torch.Tensor, block_table: torch.Tensor, q: torch.Tensor, seq_lens: torch.Tensor,
                      n_valid: Optional[torch.Tensor] = None, max_context: Optional[int] = None, out: Optional[torch.Tensor] = None,
                      seq_status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One llm42_kv4_attention call.  Returns out."""
        if q.dim() != 4 or tuple(q.shape[2:]) != (self.shape.n_q_heads, self.shape.head_dim):
            raise ValueError(f"q must be [num_seqs, window, {self.shape.n_q_heads}, {self.shape.head_dim}]")
        if max_context is None:
            max_context = block_table.shape[1] * B.LLM42_KV_BLOCK
        key = (q.shape[0], q.shape[1], max_context)
        need = self._attention4_need.get(key)
        if need is None:
            need = self._attention4_need[key] = B.llm42_kv4_attention_workspace_bytes(self.model, *key)
        if out is None:
            out = torch.zeros_like(q)
        B.llm42_kv4_attention(self.model, layer, kv4, kv4.shape[1], block_table, q, seq_lens, n_valid, max_context, out, self._room(need),
                              seq_status)
        return out

    def decode_mx4(self, kv: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, tokens: torch.Tensor,
                   kv4: Optional[torch.Tensor] = None, kv4_block_table: Optional[torch.Tensor] = None, max_context: Optional[int] = None,
                   out_tokens: Optional[torch.Tensor] = None, seq_status: Optional[torch.Tensor] = None, sampling=None) -> torch.Tensor:
        """One llm42_decode_step_mx4 call: the fast path by 4-bit weights, over the 4-bit cache if one is given.  Returns out_tokens."""
        if max_context is None:
            max_context = block_table.shape[1] * B.LLM42_KV_BLOCK
        key = (seq_lens.numel(), max_context)
        need = self._decode4_need.get(key)
        if need is None:
            need = self._decode4_need[key] = B.llm42_decode_step_mx4_workspace_bytes(self.mx4, *key)
        if out_tokens is None:
            out_tokens = torch.empty(seq_lens.numel(), dtype=torch.int32, device=self.device)
        table4 = None if kv4 is None else block_table if kv4_block_table is None else kv4_block_table
        B.llm42_decode_step_mx4(self.model, self.mx4, kv, kv.shape[2], block_table, kv4, 0 if kv4 is None else kv4.shape[1], table4, seq_lens,
                                tokens, max_context, out_tokens, self._room(need), seq_status, sampling=sampling)
        return out_tokens

    # ---- the fast path over selected blocks ----
    def paged(self, kv: torch.Tensor, bounds=True):
        """The operators around the cache `kv` of this model (paged.PagedCache)."""
        from .paged import PagedCache
        return PagedCache(kv, self.shape.n_q_heads, self.shape.head_dim, bounds)

    def decode_sparse(self, cache, block_table: torch.Tensor, seq_lens: torch.Tensor, tokens: torch.Tensor, budget: int, sink: int = 1,
                      recent: int = 2, max_context: Optional[int] = None, out_tokens: Optional[torch.Tensor] = None,
                      seq_status: Optional[torch.Tensor] = None, sampling=None) -> torch.Tensor:
        """One llm42_decode_step_sparse call: the fast path with attention over `budget` blocks; cache: what `paged` made, with the bounds of
        everything below seq_lens stored.  Returns out_tokens."""
        if max_context is None:
            max_context = block_table.shape[1] * B.LLM42_KV_BLOCK
        key = (seq_lens.numel(), max_context, budget)
        need = self._decode_sparse_need.get(key)
        if need is None:
            need = self._decode_sparse_need[key] = B.llm42_decode_step_sparse_workspace_bytes(self.model, *key)
        if out_tokens is None:
            out_tokens = torch.empty(seq_lens.numel(), dtype=torch.int32, device=self.device)
        B.llm42_decode_step_sparse(self.model, cache.heads, cache.kv, cache.num_blocks, block_table, cache.kept_bounds(), budget, sink, recent,
                                   seq_lens, tokens, max_context, out_tokens, self._room(need), seq_status, sampling=sampling)
        return out_tokens

    def commit(self, candidates: torch.Tensor, out_tokens: torch.Tensor, seq_lens: torch.Tensor,
               n_valid: Optional[torch.Tensor] = None):
        """One llm42_commit_rollback call; seq_lens is updated in place.
        Returns (committed_counts, committed_tokens, rolled_back_counts)."""
        num_seqs, window = candidates.shape
        counts = torch.empty(num_seqs, dtype=torch.int32, device=self.device)
        tokens = torch.empty((num_seqs, window), dtype=torch.int32, device=self.device)
        rolled = torch.empty(num_seqs, dtype=torch.int32, device=self.device)
        B.llm42_commit_rollback(candidates, out_tokens, n_valid, seq_lens, counts, tokens, rolled)
        return counts, tokens, rolled

    def prefill(self, kv: torch.Tensor, block_table: torch.Tensor, prompts: Sequence[np.ndarray],
                window: int = 32, cached: Optional[torch.Tensor] = None, sampling=None) -> torch.Tensor:
        """One llm42_prefill call: the prompts are appended behind the `cached` positions (int32 [n_seq] on
        the device; none by default) in passes of `window` rows per sequence.  Returns the first output
        token of each sequence (device, int32).  Raises if a sequence was flagged."""
        n_seq = len(prompts)
        lens = np.array([len(p) for p in prompts], dtype=np.int64)
        offsets = np.zeros(n_seq + 1, dtype=np.int32)
        offsets[1:] = np.cumsum(lens)
        flat = np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts]) if lens.sum() else np.zeros(1, np.int32)
        if cached is None:
            cached = torch.zeros(n_seq, dtype=torch.int32, device=self.device)
        max_context = min(block_table.shape[1] * B.LLM42_KV_BLOCK, self.cfg.max_position)
        ws = self._room(B.llm42_prefill_workspace_bytes(self.model, n_seq, window, max_context))
        first = torch.empty(n_seq, dtype=torch.int32, device=self.device)
        status = torch.empty(n_seq, dtype=torch.int32, device=self.device)
        B.llm42_prefill(self.model, kv, kv.shape[2], block_table, cached, torch.as_tensor(flat, device=self.device),
                        torch.as_tensor(offsets, device=self.device), int(lens.max()), window, max_context, first,
                        ws, status, sampling=sampling)
        if int(status.max()) != 0:
            raise RuntimeError(f"prefill: sequence status {status.tolist()}")
        return first

    def prefill_by_windows(self, kv: torch.Tensor, block_table: torch.Tensor, prompts: Sequence[np.ndarray],
                           window: int = 32) -> torch.Tensor:
        """The same prefill driven from the host through llm42_verify_window, one call per window over
        the sequences that still have prompt tokens left (what llm42_prefill must reproduce bit for bit).
        Returns the first output token of each sequence."""
        n_seq = len(prompts)
        lens = np.array([len(p) for p in prompts], dtype=np.int32)
        done = np.zeros(n_seq, dtype=np.int32)
        first = torch.full((n_seq,), -1, dtype=torch.int32, device=self.device)
        max_context = int(lens.max())
        while (done < lens).any():
            cand = np.zeros((n_seq, window), dtype=np.int32)
            nv = np.zeros(n_seq, dtype=np.int32)
            for s in range(n_seq):
                n = int(min(window, lens[s] - done[s]))
                nv[s] = n
                if n > 0:
                    cand[s, :n] = prompts[s][done[s]:done[s] + n]
            active = np.nonzero(nv > 0)[0]
            sel = torch.as_tensor(active, device=self.device)
            out, status, _ = self.verify(kv, block_table[sel].contiguous(),
                                         torch.as_tensor(done[active], device=self.device),
                                         torch.as_tensor(cand[active], device=self.device),
                                         torch.as_tensor(nv[active], device=self.device),
                                         max_context=max_context)
            if int(status.max()) != 0:
                raise RuntimeError(f"prefill: sequence status {status.tolist()}")
            done[active] += nv[active]
            fin = [j for j, s in enumerate(active) if done[s] == lens[s]]
            for j in fin:
                first[active[j]] = out[j, nv[active[j]] - 1]
        return first
