"""The chunk attention's plan, the library's own arithmetic (csrc/chunk.hpp) compiled for the CPU, over
random ragged batches: every key of every tile in one item of one queue, partial slots distinct and within
the workspace, the merge's list within its bound, and no item so long that the device would wait for it."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_31315_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "chunk_plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so,
                    os.path.join(HERE, "chunk_plan_check.cpp")], check=True)
    return ctypes.CDLL(so)


def _run(plan, Hkv, G, causal, ctx, B, slots=1024):
    c, b = (np.ascontiguousarray(x, np.int32) for x in (ctx, B))
    items, pieces, largest = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_double(0)
    line = plan.check_chunk(len(c), Hkv, G, causal, c.ctypes.data_as(ctypes.c_void_p), b.ctypes.data_as(ctypes.c_void_p),
                            slots, ctypes.byref(items), ctypes.byref(pieces), ctypes.byref(largest))
    assert line == 0, f"chunk_plan_check.cpp:{line}"
    return items.value, pieces.value, largest.value


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("seed", range(10))
def test_ragged(plan, seed, causal):
    rng = np.random.default_rng(seed)
    for _ in range(12):
        S, Hkv, G = int(rng.integers(1, 80)), int(rng.choice([1, 2, 3, 4, 8, 16])), int(rng.choice([1, 4, 5, 7, 8, 32, 200, 256]))
        B = rng.integers(0, int(rng.choice([2, 70, 500, 3000])), S)
        B[rng.random(S) < 0.2] = rng.integers(0, 2)
        _run(plan, Hkv, G, causal, rng.integers(0, int(rng.choice([1, 300, 3000, 70000])), S), B, int(rng.choice([0, 2, 64, 1024])))


@pytest.mark.parametrize("S,Hkv,G,ctx,B", [(1, 8, 4, 0, 8192), (1, 4, 8, 65536, 2048), (8, 8, 4, 3000, 800), (1, 8, 4, 500, 100),
                                           (1, 1, 256, 0, 1500), (1, 8, 4, 0, 131072), (1, 64, 1, 1 << 20, 4096), (300, 8, 4, 4000, 1)])
def test_no_item_is_long(plan, S, Hkv, G, ctx, B):
    """Where a batch's work is spread evenly, the longest item is no longer than 1.6 workgroups' even share, or one that
    cannot be cut (128 + 256 keys at least; large counts of tiles are left whole)."""
    _, _, largest = _run(plan, Hkv, G, 1, [ctx] * S, [B] * S)
    share = 8 * (128 + 2 * 256)
    units = S * Hkv * -(-B * G // 256) * (ctx + B + 128) * 8 / 256
    assert largest < 1.6 or largest * units < 2 * share


@pytest.mark.parametrize("S,ctx,B", [(1, 4000, 400), (2, 1800, 200), (2, 4000, 200)])
def test_the_last_tiles_of_small_batches_are_cut_too(plan, S, ctx, B):
    """A tile of 64 rows takes three quarters of a full one's time."""
    items, pieces, _ = _run(plan, 8, 4, 1, [ctx] * S, [B] * S)
    assert items == pieces > 0


def test_empty(plan):
    assert _run(plan, 8, 4, 1, [5, 0], [0, 0]) == (0, 0, 0.0)
