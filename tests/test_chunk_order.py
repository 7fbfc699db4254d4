"""The order in which the chunk attention's plan takes a batch's sequences, and the plan in that order, from the
arithmetic that the device runs (csrc/chunk.hpp) compiled for the CPU: batches that mix sequences of few rows with
others, with empty ones, equal ones, and more than the plan orders."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_31315_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("order") / "chunk_order.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so,
                    os.path.join(HERE, "chunk_order_check.cpp")], check=True)
    return ctypes.CDLL(so)


def _run(plan, Hkv, G, causal, ctx, B, slots=1024):
    c, b = (np.ascontiguousarray(x, np.int32) for x in (ctx, B))
    order = np.zeros(len(c), np.int32)
    longest, share, dropped = ctypes.c_double(0), ctypes.c_double(0), ctypes.c_int(0)
    line = plan.check_order(len(c), Hkv, G, causal, *(x.ctypes.data_as(ctypes.c_void_p) for x in (c, b)), slots,
                            order.ctypes.data_as(ctypes.c_void_p), ctypes.byref(longest), ctypes.byref(share),
                            ctypes.byref(dropped))
    assert line == 0, f"chunk_order_check.cpp:{line}"
    return order, longest.value, share.value, dropped.value


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("seed", range(8))
def test_mixed_batches(plan, seed, causal):
    rng = np.random.default_rng(seed)
    for _ in range(12):
        S, Hkv, G = int(rng.integers(1, 200)), int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 4, 5, 8, 64, 65, 256]))
        B = np.where(rng.random(S) < rng.random(), 1, rng.integers(0, int(rng.choice([70, 500, 3000])), S))
        B[rng.random(S) < 0.1] = 0
        ctx = rng.integers(0, int(rng.choice([1, 300, 3000, 70000])), S)
        _run(plan, Hkv, G, causal, ctx, B, int(rng.choice([0, 2, 64, 1024])))


@pytest.mark.parametrize("S", [1, 63, 64, 65, 128, 1024, 1025, 1300])
def test_rounds(plan, S):
    """Numbers of sequences about the plan's rounds of 64 and the most that it orders; all alike, so ties keep their order."""
    rng = np.random.default_rng(S)
    order, *_ = _run(plan, 2, 4, 1, [100] * S, [90] * S)
    assert (order == np.arange(S)).all()
    _run(plan, 2, 4, 1, rng.integers(0, 2000, S), np.where(rng.random(S) < 0.7, 1, rng.integers(0, 400, S)))


def test_few_rows_are_spread_among_the_others(plan):
    """Eight prompt chunks and 24 single tokens, all alike within their kind: three tokens to a chunk."""
    ctx, B = [4000] * 32, [1000] * 8 + [1] * 24
    order, *_ = _run(plan, 8, 4, 1, ctx, B)
    where = [r for r, s in enumerate(order) if s < 8]
    assert [b - a for a, b in zip(where, where[1:])] == [4] * 7


@pytest.mark.parametrize("S,tokens,ctx,B", [(32, 24, 16000, 2000), (64, 60, 30000, 800), (8, 4, 3000, 300), (200, 190, 8000, 500),
                                            (16, 8, 60000, 100), (33, 32, 1000, 4000)])
def test_no_item_of_a_mixed_batch_is_long(plan, S, tokens, ctx, B):
    """Tiles stay whole up to a 128th of the batch's work, two workgroups' shares.  Longer ones are cut into what fits the
    device, no piece above two shares and what cutting costs (512 keys of 8 units), but for pieces of 512 to 1024 keys and a
    step's rounding, with 128 keys for an item."""
    rng = np.random.default_rng(S)
    rows = np.array([B] * (S - tokens) + [1] * tokens)
    _, longest, share, dropped = _run(plan, 8, 4, 1, rng.integers(ctx // 2, ctx + 1, S), rows)
    assert dropped == 0
    assert longest <= max(2 * share + 8 * 512, 8 * 1024) + 8 * (64 + 128)


def test_no_rows_at_all(plan):
    order, longest, *_ = _run(plan, 8, 4, 1, [5, 0, 7], [0, 0, 0])
    assert list(order) == [0, 1, 2] and longest == 0
