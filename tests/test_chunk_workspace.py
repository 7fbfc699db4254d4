"""The workspace that sd_chunk_attn_paged asks for, on the host: within the documented bound whatever the shape."""
import ctypes
import random

import pytest

from paper_2606_31315_amd import _lib as L


def need(S, Hq, Hkv, D, max_ctx, max_block, total_q=None, Lmax=None):
    sh = L.SdAttnShape(S, Hq, Hkv, D, Lmax or max_ctx + max_block, S * max_block if total_q is None else total_q, max_ctx,
                       max_block, L.SD_BF16, 0.0)
    n = ctypes.c_size_t(0)
    assert L.lib().sd_chunk_attn_workspace_size(ctypes.byref(sh), ctypes.byref(n)) == L.SD_OK, (S, Hq, Hkv, D, max_ctx, max_block)
    return n.value


def bound(S, Hkv, D):
    return {128: 137_000_000, 64: 70_000_000}[D] + 48 * S + 4 * S * Hkv


@pytest.mark.parametrize("S,max_ctx,max_block", [(256, 32000, 32), (512, 65000, 32), (1024, 131000, 1), (32, 16000, 16), (20000, 400, 4),
                                                 (8192, 130000, 16), (1, 2 ** 31 - 600, 64)])
@pytest.mark.parametrize("D", [64, 128])
def test_many_sequences_of_short_blocks(S, max_ctx, max_block, D):
    assert need(S, 32, 8, D, max_ctx, max_block) <= bound(S, 8, D)


def test_random_shapes():
    rng = random.Random(1)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))  # noqa: E731
    for _ in range(4000):
        S, Hkv, G, D = log(1, 30000), rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 2, 4, 7, 8, 16, 64, 256]), rng.choice([64, 128])
        max_ctx, max_block = log(1, 200000), rng.choice([1, log(1, 64), log(1, 8192)])
        total = log(1, min(S * max_block, 1 << 24))
        assert need(S, G * Hkv, Hkv, D, max_ctx, max_block, total) <= bound(S, Hkv, D), (S, Hkv, G, D, max_ctx, max_block, total)
