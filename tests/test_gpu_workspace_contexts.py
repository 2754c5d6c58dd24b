"""llm42_workspace_bytes serves calls of every context up to max_context, although a shorter one may split its attention finer: per chunk of 256 keys, where the
longest runs per 2048, or a wave per chunk."""
import numpy as np
import pytest
import torch

from helpers import wl
from gpu_helpers import VerifierSession
from paper_2601_17768_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPE = wl.TINY.replace(d_model=512, n_q_heads=32, n_kv_heads=8, head_dim=128)


@pytest.fixture(scope="module")
def sess():
    s = VerifierSession(SHAPE, wl.make_weights(SHAPE, seed=58), max_position=60000, device=DEV)
    yield s
    s.close()


@pytest.mark.parametrize("window", [1, 4, 13, 64])
@pytest.mark.parametrize("max_seqs", [1, 3, 24, 130])
def test_the_size_does_not_fall_where_the_context_grows(sess, max_seqs, window):
    contexts = sorted({c + d for c in list(range(2048, 60000, 2048)) + [256, 512, 1024, 1152, 1280, 1536] for d in (-1, 0, 1)} | {64, 60000})
    sizes = [B.llm42_workspace_bytes(sess.model, max_seqs, window, c) for c in contexts if c >= window]
    assert sizes == sorted(sizes)
    assert sizes[-1] <= B.llm42_workspace_bytes(sess.model, max_seqs + 1, window, 60000)


@pytest.mark.parametrize("num,longest,shorter", [(3, 16384, 14336), (1, 49152, 47104), (2, 24576, 22528)])
def test_a_workspace_for_the_longest_context_serves_a_shorter_one(sess, num, longest, shorter):
    """8 kv heads, one token: from 192 workgroups of 2048 keys on a call has one each, below that one for every 256."""
    ws = torch.empty(B.llm42_workspace_bytes(sess.model, num, 1, longest), dtype=torch.uint8, device=DEV)
    blocks = num * 5 + 1
    kv = sess.kv_cache(blocks)
    kv.normal_(generator=torch.Generator(device=DEV).manual_seed(3))
    table = np.full((num, longest // 16), -1, np.int32)
    table[:, :5] = np.arange(num * 5).reshape(num, 5)
    d = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32), device=DEV)
    outs = []
    for c in (longest, shorter, 80):
        out = torch.full((num, 1), -7, dtype=torch.int32, device=DEV)
        B.llm42_verify_window(sess.model, kv, blocks, d(table), d([70] * num), d([[5]] * num), 1, None, c, out, ws)
        outs.append(out)
    assert int(outs[0].min()) >= 0 and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
