"""The operators around the paged bf16 cache (include/llm42_paged.h): handles, buffers and their sizes around the binding's calls.  No arithmetic
happens here.

A decoder layer's attention by these, for models whose heads are normed or rotated in other ways than llm42.h's, or whose fast path reads a part of
the context:

    cache.append(layer, k, v, table, lens, q=q, q_out=q, rope=rope, q_norm=gq, k_norm=gk)
    lists = cache.select(layer, q, table, lens, budget=64)
    out = cache.attention(layer, q, table, lens, lists)

Workspaces come from torch's allocator, one for each call that needs one: calls on different streams and captured graphs share none.
What a captured graph reads and writes (the Rope and the PagedCache among it) is kept by whoever keeps the graph.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple, Union

import torch

from . import binding as B

_LAYOUTS = {"half": B.LLM42_ROPE_HALF, "interleaved": B.LLM42_ROPE_INTERLEAVED}
_SCALINGS = {"none": (B.LLM42_ROPE_NONE, ()),
             "linear": (B.LLM42_ROPE_LINEAR, ("factor",)),
             "llama3": (B.LLM42_ROPE_LLAMA3, ("factor", "low_freq_factor", "high_freq_factor", "original_max_position")),
             "yarn": (B.LLM42_ROPE_YARN, ("factor", "beta_fast", "beta_slow", "original_max_position"))}
_dropped = []           # (device, handle) of tables whose owner went away without closing them


def _give_back_dropped():
    while _dropped:
        device, handle = _dropped.pop()
        torch.cuda.synchronize(device)
        B.llm42_rope_destroy(handle)


class Rope:
    """Rotary positions on the current device: the first rot_dim features of a head, in pairs by `layout` ("half": j and j + rot_dim / 2, "interleaved":
    2 j and 2 j + 1), frequencies theta^(-2 j / rot_dim) scaled by `scaling`: a dict with "kind" ("none", "linear", "llama3", "yarn"), the kind's
    parameters by their names in llm42_rope_config, and if it is not the kind's own, attention_factor.

    A table holds 4 * rot_dim bytes a position until close(), which waits for its device, as making one does: neither belongs in a capture, on whatever stream.
    One that is dropped instead is given back where the next is made or closed: a finalizer runs at any time, and frees and waits for nothing."""

    def __init__(self, rot_dim: int, theta: float, max_position: int, layout: str = "half", scaling: Optional[Dict] = None):
        self.handle = None
        if layout not in _LAYOUTS:
            raise ValueError(f"unknown layout {layout!r}")
        given = dict(scaling or {"kind": "none"})
        kind = given.pop("kind", None)
        if kind not in _SCALINGS:
            raise ValueError(f"unknown scaling {kind!r}")
        number, names = _SCALINGS[kind]
        if not set(names) <= set(given) <= set(names) | {"attention_factor"}:
            raise ValueError(f"scaling {kind!r} takes {', '.join(names) or 'nothing'} (and attention_factor), got {', '.join(given) or 'nothing'}")
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a rotary table must be made before a capture")
        _give_back_dropped()
        self.rot_dim, self.max_position, self.device = rot_dim, max_position, torch.cuda.current_device()
        self.handle = B.llm42_rope_create(B.RopeConfig(rot_dim=rot_dim, layout=_LAYOUTS[layout], scaling=number, max_position=max_position,
                                                       theta=theta, **given))

    def close(self):
        if self.handle:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a rotary table must be closed outside of a capture")
            _dropped.append((self.device, self.handle))
            self.handle = None
            _give_back_dropped()

    def __del__(self):
        if getattr(self, "handle", None) and _dropped is not None:      # (None while the interpreter ends)
            _dropped.append((self.device, self.handle))
            self.handle = None


class PagedCache:
    """A paged bf16 cache [n_layers, 2, num_blocks, n_kv_heads, 16 * head_dim] (kv_layout.alloc_kv, VerifierSession.kv_cache) and, if bounds are asked for
    (True, or a uint8 tensor that holds them), the bounds of its keys."""

    def __init__(self, kv: torch.Tensor, n_q_heads: int, head_dim: int, bounds: Union[bool, torch.Tensor] = True):
        if kv.dim() != 5 or kv.shape[1] != 2 or kv.shape[4] != 16 * head_dim or kv.dtype != torch.bfloat16:
            raise ValueError("kv must be bfloat16 [n_layers, 2, num_blocks, n_kv_heads, 16 * head_dim]")
        self.kv, self.num_blocks = kv, kv.shape[2]
        self.heads = B.Heads(kv.shape[0], n_q_heads, kv.shape[3], head_dim)
        need = B.llm42_kv_bounds_bytes(self.heads, self.num_blocks)
        if isinstance(bounds, torch.Tensor):
            self.bounds = bounds
        else:
            self.bounds = torch.empty(need, dtype=torch.uint8, device=kv.device) if bounds else None
        self._select_need: Dict = {}
        self._attention_need: Dict = {}

    def kept_bounds(self) -> torch.Tensor:
        if self.bounds is None:
            raise ValueError("the cache was made without bounds")
        return self.bounds

    @staticmethod
    def _room(block_table: torch.Tensor, max_context: Optional[int], rope: Optional[Rope] = None) -> int:
        if max_context is None:
            max_context = block_table.shape[1] * B.LLM42_KV_BLOCK
            if rope is not None:
                max_context = min(max_context, rope.max_position)
        return max_context

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, n_valid: Optional[torch.Tensor] = None,
               max_context: Optional[int] = None, rope: Optional[Rope] = None, q_norm: Optional[torch.Tensor] = None,
               k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, seq_status: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """One llm42_kv_append call; the bounds of blocks that become whole are kept up if the cache has bounds.  Returns q_out (zeros where a row takes no part,
        unless it is given)."""
        if rope is not None and not rope.handle:
            raise ValueError("the rotary table is closed")
        if q is not None and q_out is None:
            q_out = torch.zeros(q.shape, dtype=torch.bfloat16, device=q.device)
        B.llm42_kv_append(self.heads, layer, self.kv, self.num_blocks, block_table, self.bounds, q, k, v, q_norm, k_norm, eps,
                          None if rope is None else rope.handle, seq_lens, n_valid, self._room(block_table, max_context, rope), q_out, seq_status)
        return q_out

    def store_bounds(self, block_table: torch.Tensor, first: torch.Tensor, count: torch.Tensor, max_count: int, layer: int = -1,
                     seq_status: Optional[torch.Tensor] = None) -> None:
        """One llm42_kv_bounds_store call: behind a prefill, or a verifier pass and its commit."""
        B.llm42_kv_bounds_store(self.heads, layer, self.kv, self.num_blocks, block_table, self.kept_bounds(), first, count, max_count, seq_status)

    def read_bounds(self, block_ids: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """One llm42_kv_bounds_read call: (smallest, largest) of the physical blocks, bfloat16 [n_layers, len(block_ids), n_kv_heads, head_dim];
        zeros where an id is out of range."""
        h = self.heads
        lo, hi = (torch.empty((h.n_layers, block_ids.numel(), h.n_kv_heads, h.head_dim), dtype=torch.bfloat16, device=self.kv.device)
                  for _ in range(2))
        B.llm42_kv_bounds_read(h, self.kept_bounds(), self.num_blocks, block_ids, lo, hi)
        return lo, hi

    def select(self, layer: int, q: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, budget: int, sink: int = 1, recent: int = 2,
               n_valid: Optional[torch.Tensor] = None, max_context: Optional[int] = None, selected: Optional[torch.Tensor] = None,
               seq_status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One llm42_kv_select call.  Returns the lists, int32 [num_seqs, window, n_kv_heads, budget] (-1 where a row takes no part, unless they are given)."""
        shape = (*q.shape[:2], self.heads.n_kv_heads, budget)
        if selected is None:
            selected = torch.full(shape, -1, dtype=torch.int32, device=q.device)
        if tuple(selected.shape) != shape:
            raise ValueError(f"selected must be {list(shape)}")
        max_context = self._room(block_table, max_context)
        key = (shape[0], shape[1], max_context, budget)
        need = self._select_need.get(key)
        if need is None:
            need = self._select_need[key] = B.llm42_kv_select_workspace_bytes(self.heads, *key)
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        B.llm42_kv_select(self.heads, layer, self.num_blocks, block_table, self.kept_bounds(), q, seq_lens, n_valid, max_context, sink, recent,
                          selected, ws, seq_status)
        return selected

    def attention(self, layer: int, q: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, selected: torch.Tensor,
                  n_valid: Optional[torch.Tensor] = None, max_context: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  scale: float = 0.0, seq_status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One llm42_kv_sparse_attention call.  Returns out (zeros where a row takes no part, unless it is given)."""
        if out is None:
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        key = (q.shape[0], q.shape[1], selected.shape[-1])
        need = self._attention_need.get(key)
        if need is None:
            need = self._attention_need[key] = B.llm42_kv_sparse_attention_workspace_bytes(self.heads, *key)
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        B.llm42_kv_sparse_attention(self.heads, layer, self.kv, self.num_blocks, block_table, q, seq_lens, n_valid,
                                    self._room(block_table, max_context), selected, scale, out, ws, seq_status)
        return out
