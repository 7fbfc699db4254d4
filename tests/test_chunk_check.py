"""sd_check_chunk_inputs: the error word for the lengths that sd_chunk_attn_paged takes on trust, which allow more than
the block attention's (any number of rows, bounds whose sum exceeds the cache, rows behind the last sequence)."""
import ctypes

import numpy as np
import pytest
import torch

import gpu_util as G
import paper_2606_31315_amd as sd
from paper_2606_31315_amd import _lib as L

P = ctypes.c_void_p
CTX, BLOCK, OFFSETS = 1, 2, 4


def shape(**kw):
    sh = L.SdAttnShape(4, 32, 8, 128, 4096, 900, 3000, 2000, L.SD_BF16, 0.0)
    for k, v in kw.items():
        setattr(sh, k, v)
    return sh


@pytest.mark.parametrize("field,value", [("num_seqs", -1), ("total_q", -1), ("max_kv_len", 0), ("max_ctx", -1), ("max_ctx", 4097),
                                         ("max_block", 0), ("max_block", 4097)])
def test_shape_errors(field, value):
    assert L.lib().sd_check_chunk_inputs(ctypes.byref(shape(**{field: value})), *map(P, (16, 32, 48, 64)), None) == L.SD_ERR_INVALID_ARG
    assert L.lib().sd_last_error().decode().startswith("sd_check_chunk_inputs")


def test_pointer_errors():
    call = L.lib().sd_check_chunk_inputs
    assert call(None, *map(P, (16, 32, 48, 64)), None) == L.SD_ERR_INVALID_ARG
    for i in range(4):
        p = [16, 32, 48, 64]
        p[i] = None
        assert call(ctypes.byref(shape()), *map(P, p), None) == L.SD_ERR_INVALID_ARG, i


def test_binding_shapes():
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="meta")  # noqa: E731
    kw = dict(total_q=9, max_ctx=32, max_chunk=8, max_kv_len=64)
    with pytest.raises(ValueError, match="^ctx_lens has shape"):
        sd.check_chunk_inputs(i32(4), i32(3), i32(4), **kw)
    with pytest.raises(ValueError, match="^q_offsets has shape"):
        sd.check_chunk_inputs(i32(3), i32(3), i32(3), **kw)
    with pytest.raises(ValueError, match="^status has shape"):
        sd.check_chunk_inputs(i32(3), i32(3), i32(4), status=i32(2), **kw)
    with pytest.raises(ValueError, match="device tensor"):
        sd.check_chunk_inputs(i32(3), i32(3), i32(4), **kw)


def _status(ctx, B, off, total_q, max_ctx=3000, max_chunk=2000, max_kv_len=4096):
    t = [torch.from_numpy(np.asarray(x, np.int32)).to(G.dev()) for x in (ctx, B, off)]
    G.log(f"sd_check_chunk_inputs S={len(B)} total_q={total_q} max_ctx={max_ctx} max_chunk={max_chunk} keys={max_kv_len}")
    st = sd.check_chunk_inputs(*t, total_q=total_q, max_ctx=max_ctx, max_chunk=max_chunk, max_kv_len=max_kv_len)
    torch.cuda.synchronize()
    return st.cpu().tolist()


CTX_OK, B_OK = [3000, 0, 2096, 17], [1000, 65, 2000, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("pad", [0, 1, 500])
def test_sound_lengths(pad):
    off = np.concatenate([[0], np.cumsum(B_OK)])
    assert _status(CTX_OK, B_OK, off, off[-1] + pad) == [0, -1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("what,seq,value,bits", [
    ("ctx", 0, 3001, CTX), ("ctx", 1, -1, CTX), ("ctx", 2, 2097, CTX), ("ctx", 1, 2 ** 31 - 1, CTX),
    ("B", 2, 2001, BLOCK | OFFSETS), ("B", 3, -1, BLOCK | OFFSETS), ("B", 1, 64, OFFSETS), ("B", 1, 2 ** 31 - 1, BLOCK | OFFSETS),
    ("off", 0, 1, OFFSETS), ("off", 1, 999, OFFSETS), ("off", 4, 3064, OFFSETS)])
def test_each_fault(what, seq, value, bits):
    x = {"ctx": np.array(CTX_OK), "B": np.array(B_OK), "off": np.concatenate([[0], np.cumsum(B_OK)])}
    total = int(x["off"][-1])
    x[what][seq] = value
    st = _status(x["ctx"], x["B"], x["off"], total)
    assert st[0] == bits and st[2] >= 1 and st[1] == (seq - 1 if what == "off" and seq else seq)


@pytest.mark.gpu
def test_too_few_rows():
    """The last sequences end behind the rows that there are."""
    off = np.concatenate([[0], np.cumsum(B_OK)])
    assert _status(CTX_OK, B_OK, off, 1065) == [OFFSETS, 2, 2]


@pytest.mark.gpu
def test_no_sequences():
    assert _status([], [], [0], 7) == [0, -1, 0]
