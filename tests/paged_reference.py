"""The operators around the paged bf16 cache by their definitions, in float64 on the CPU, one head and one row at a time."""
import math

import torch


def frequencies(rot, theta, scaling):
    """(angle per position of every pair, attention factor), from wavelengths rather than turns."""
    kind = scaling.get("kind", "none")
    out = []
    factor = scaling.get("attention_factor") or (0.1 * math.log(scaling["factor"]) + 1.0 if kind == "yarn" else 1.0)
    for j in range(rot // 2):
        f = math.exp(-2.0 * j / rot * math.log(theta))
        if kind == "linear":
            f /= scaling["factor"]
        elif kind == "llama3":
            n, wave = scaling["original_max_position"], 2 * math.pi / f
            short, long_ = n / scaling["high_freq_factor"], n / scaling["low_freq_factor"]
            if wave > long_:
                f /= scaling["factor"]
            elif wave > short:
                x = (n / wave - scaling["low_freq_factor"]) / (scaling["high_freq_factor"] - scaling["low_freq_factor"])
                f = (1 - x) * f / scaling["factor"] + x * f
        elif kind == "yarn":
            at = lambda turns: rot * math.log(scaling["original_max_position"] / (turns * 2 * math.pi)) / (2 * math.log(theta))
            lo, hi = max(math.floor(at(scaling["beta_fast"])), 0), min(math.ceil(at(scaling["beta_slow"])), rot - 1)
            ramp = min(max((j - lo) / ((hi if hi != lo else hi + 0.001) - lo), 0.0), 1.0)
            f = f / scaling["factor"] * ramp + f * (1 - ramp)
        out.append(f)
    return out, factor


def turned(x, pos, gain, eps, rope):
    """x [..., head_dim] at one position; rope: None or (rot_dim, theta, layout, scaling)."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if rope is None:
        return x
    rot, theta, layout, scaling = rope
    freq, factor = frequencies(rot, theta, scaling)
    y = x.clone()
    for j, f in enumerate(freq):
        a, b = (j, j + rot // 2) if layout == "half" else (2 * j, 2 * j + 1)
        c, s = math.cos(pos * f) * factor, math.sin(pos * f) * factor
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def exponent(top):
    e = -40
    while top > 127 * 2.0 ** e:
        e += 1
    return e


def bounds(k):
    """k [16, head_dim] -> (smallest, largest) float64, infinite where the block's are."""
    k = k.double()
    top = float(k.abs().max())
    if not bool(torch.isfinite(k).all()) or top > 127 * 2.0 ** 40:
        inf = torch.full((k.shape[1],), math.inf, dtype=torch.float64)
        return -inf, inf
    unit = 2.0 ** exponent(top)
    return torch.floor(k.amin(0) / unit) * unit, torch.ceil(k.amax(0) / unit) * unit


def rounded_query(q):
    q = q.double()
    if not bool(torch.isfinite(q).all()) or float(q.abs().max()) > 127 * 2.0 ** 40:
        return torch.zeros_like(q)
    unit = 2.0 ** exponent(float(q.abs().max()))
    return torch.round(q / unit) * unit


def select(q, lo, hi, own, budget, sink, recent):
    """q [group, head_dim], lo / hi [blocks, head_dim] -> the selected blocks of a row, ascending, -1 behind them."""
    if own + 1 <= budget:
        ids = list(range(own + 1))
    else:
        forced = list(range(sink)) + list(range(own + 1 - recent, own + 1))
        between = [b for b in range(sink, own + 1 - recent)]
        at = torch.tensor(between, dtype=torch.long)
        infinite = torch.isinf(hi[at]).any(-1)
        l, h = (torch.where(infinite[:, None], 0.0, x[at]) for x in (lo, hi))
        qr = torch.stack([rounded_query(x) for x in q])
        score = torch.maximum(qr[:, None] * l, qr[:, None] * h).sum(-1).amax(0)
        score = torch.where(infinite, math.inf, score).tolist()
        best = sorted(range(len(between)), key=lambda i: (-score[i], i))[:budget - len(forced)]
        ids = sorted(forced + [between[i] for i in best])
    return ids + [-1] * (budget - len(ids))


def attention(q, k, v, blocks, pos, scale):
    """One row: q [group, head_dim], k / v [tokens, head_dim], blocks: list entries.  Returns (output, sum of weights times |v|)."""
    keys = [p for b in blocks if 0 <= b <= pos // 16 for p in range(16 * b, min(16 * b + 16, pos + 1))]
    if not keys:
        return torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    at = torch.tensor(keys)
    p = torch.softmax(q.double() @ k[at].double().t() * scale, -1)
    return p @ v[at].double(), p @ v[at].double().abs()
