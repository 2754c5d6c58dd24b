"""MXFP4 and attention over a cache held in it, in 64 bits and from the definition: what the 4-bit operators are compared with."""
from __future__ import annotations

import math

import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantized(x: torch.Tensor) -> torch.Tensor:
    """The values that x stands for in MXFP4, blocks of 32 along the last axis, float64."""
    n = x.shape[-1]
    d = torch.nn.functional.pad(x.double(), (0, -n % 32)).unflatten(-1, (-1, 32))
    top = d.abs().max(-1, keepdim=True).values
    finite = torch.isfinite(d).all(-1, keepdim=True)
    e = (torch.floor(torch.log2(torch.where(finite, top, 1.0))) - 2).clamp(-127, 127)
    m = d.abs() / torch.exp2(e)
    dist = (m[..., None] - LEVELS).abs()                                    # nearest level, the even index on a tie
    best = dist.min(-1, keepdim=True).values
    even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    pick = even_first[(dist[..., even_first] == best).int().argmax(-1)]
    out = torch.where(finite, torch.sign(d) * LEVELS[pick] * torch.exp2(e), math.nan)
    return out.flatten(-2)[..., :n]


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, first: int):
    """q [rows, heads, hd] at positions first, first + 1, ...; k, v [keys, kv heads, hd].  Returns the output and, for tolerances, the
    weighted mean of |v|."""
    n, heads, hd = q.shape
    group = heads // k.shape[1]
    out, mag = torch.empty_like(q), torch.empty_like(q)
    hidden = torch.arange(k.shape[0]) > first + torch.arange(n)[:, None]
    for h in range(heads):
        s = (q[:, h] @ k[:, h // group].T) / math.sqrt(hd)
        p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
        vh = torch.where(hidden.all(0)[:, None], 0.0, v[:, h // group])
        out[:, h], mag[:, h] = p @ vh, p @ vh.abs()
    return out, mag


class QuantizingKV:
    """A cache for the oracle's forward pass that holds what is written to it in MXFP4."""

    class Plane:
        def __init__(self, shape):
            self.t = torch.zeros(shape, dtype=torch.float64)

        def __setitem__(self, at, value):
            self.t[at] = quantized(value)

        def __getitem__(self, at):
            return self.t[at]

    def __init__(self, cfg, capacity: int):
        shape = (cfg.n_layers, capacity, cfg.n_kv_heads, cfg.head_dim)
        self.k, self.v, self.capacity = self.Plane(shape), self.Plane(shape), capacity


def quantized_weights(w: dict) -> dict:
    """A model's weights as its 4-bit copy stands for them (every value is a bf16): all matrices but the embedding."""
    q = lambda t: quantized(t).to(torch.bfloat16)
    return {"embed": w["embed"], "final_norm": w["final_norm"], "lm_head": q(w["lm_head"]),
            "layers": [{n: t if n.endswith("norm") else q(t) for n, t in lw.items()} for lw in w["layers"]]}
