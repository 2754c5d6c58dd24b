"""Rollback and recomputation statistics of the decode - verify - rollback loop (the quantities of the
paper's rollback / recompute table, section 5.1) on seeded synthetic prompts and random-init weights.

    python -m paper_2601_17768_amd.dvr_stats [--layers 32] [--groups 1,8,24] [--windows 16,32,64] [--new 128]
        [--fast bf16|mx4|mx4_cache]

For every (group size, window) the loop of paper_2601_17768_amd/dvr.py generates `--new` tokens per
sequence: fast-path candidates from llm42_decode_step (whose reduction order follows the group size; with
`--fast mx4` or `mx4_cache` from llm42_decode_step_mx4, on 4-bit weights and the bf16 or a 4-bit cache),
verification by llm42_verify_window, commit by llm42_commit_rollback.  Reported per configuration:
windows verified, windows with a rollback, candidates recomputed (count and share of all fast-path
tokens), and whether the committed stream of sequence 0 equals the one it gets when it runs alone -
the paper's claim, which must hold in every line.  With random-init weights the gap between the
two best logits of a row is much smaller than in a trained model, so the fast path's low-bit
differences flip tokens far more often than the paper's 0-11 % of recomputed tokens: the numbers
describe this implementation on this input, not the paper's workloads.  One JSON line at the end.
"""
from __future__ import annotations

import argparse
import json
import sys
import time

import numpy as np
import torch

from . import dvr
from . import workloads as wl
from .session import VerifierSession


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--groups", default="1,8,24")
    ap.add_argument("--windows", default="16,32,64")
    ap.add_argument("--new", type=int, default=128, help="tokens to commit per sequence")
    ap.add_argument("--prompt", default="32,256", help="prompt lengths: uniform in [lo, hi]")
    ap.add_argument("--fast", choices=dvr.FAST_PATHS, default="bf16", help="the fast path's weights and cache")
    args = ap.parse_args()
    groups = [int(x) for x in args.groups.split(",")]
    windows = [int(x) for x in args.windows.split(",")]
    lo, hi = (int(x) for x in args.prompt.split(","))
    shape = wl.LLAMA_8B.replace(n_layers=args.layers)
    weights = wl.make_weights(shape, seed=42)
    max_position = hi + args.new + 3 * max(windows) + 16
    sess = VerifierSession(shape, weights, max_position=max_position, device="cuda:0")
    dev = sess.device
    rng = wl.rng_for(42, 9)
    prompts = [wl.random_tokens(rng, int(n), shape.vocab) for n in wl.uniform_lengths(rng, max(groups), lo, hi)]

    def state(group):
        lens = np.array([len(p) for p in group], dtype=np.int32)
        table, num_blocks = wl.make_block_table(wl.rng_for(42, 10, len(group)), lens + args.new + 3 * max(windows), 16,
                                                spare_blocks=2)
        kv = sess.kv_cache(num_blocks)
        bt = torch.as_tensor(table, device=dev)
        first = sess.prefill(kv, bt, group, window=64)
        return kv, bt, torch.as_tensor(lens, device=dev), first

    rows = []
    alone = {}
    for window in windows:
        for g in groups:
            kv, bt, lens, first = state(prompts[:g])
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            toks, st = dvr.generate(sess, kv, bt, lens, first, args.new, window, fast=args.fast)
            torch.cuda.synchronize()
            dt = time.perf_counter() - t0
            if g == 1:
                alone[window] = toks[0]
            same = bool(torch.equal(toks[0], alone[window])) if window in alone else None
            row = {"window": window, "group": g, "windows_verified": st.iterations * g, "windows_rolled_back": st.rollbacks,
                   "fast_path_tokens": st.fast_tokens, "recomputed_tokens": st.rolled_back,
                   "recomputed_share": round(st.rolled_back / max(1, st.fast_tokens), 4),
                   "committed_tokens": st.committed, "committed_per_s": round(st.committed / dt, 1),
                   "stream_equals_alone": same}
            rows.append(row)
            print(f"window {window:3d} group {g:3d}: {row['windows_verified']:4d} windows, {st.rollbacks:4d} rolled back, "
                  f"{st.rolled_back:5d} of {st.fast_tokens:6d} candidates recomputed ({100 * row['recomputed_share']:5.2f} %), "
                  f"{row['committed_per_s']:8.1f} committed tokens/s, stream of sequence 0 as alone: {same}",
                  file=sys.stderr, flush=True)
            del kv
    sess.close()
    ok = all(r["stream_equals_alone"] in (True, None) for r in rows)
    print(json.dumps({"n_layers": args.layers, "new_tokens": args.new, "fast": args.fast, "rows": rows, "all_streams_equal": ok}), flush=True)
    if not ok:
        sys.exit("a committed stream depended on the group")


if __name__ == "__main__":
    main()
