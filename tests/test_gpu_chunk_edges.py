"""sd_chunk_attn_paged at the edges of its tiles, pieces and contract."""
import numpy as np
import pytest
import torch

import gpu_util as G
import paper_2606_31315_amd as sd
import prefill_ref as R

pytestmark = pytest.mark.gpu
CAUSAL, BIDIR = R.CAUSAL, R.BIDIR


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(G.dev())


def _run(b, mask, **kw):
    kw.setdefault("max_ctx", int(b["ctx"].max()))
    kw.setdefault("max_chunk", max(1, int(b["B"].max())))
    G.log(f"sd_chunk_attn_paged q={list(b['q'].shape)} pool={list(b['kp'].shape)} ctx={b['ctx'][:8].tolist()} "
          f"B={b['B'][:8].tolist()} mask={mask}")
    o = sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], _i32(b["ctx"]), _i32(b["B"]), _i32(b["off"]), mask, **kw)
    torch.cuda.synchronize()
    return o


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx,B,first,keys", [(20000, 100, 4096, 4096), (20000, 4, 4096, 4096), (500, 100, 64, 256), (500, 250, 64, 64)],
                         ids=["pieces", "splits", "halves", "tiles"])
def test_keys_that_are_no_numbers_reach_every_row(ctx, B, first, keys, D):
    """A run of NaN keys longer than a piece, a split or a tile: no row's result is made from the rest alone."""
    b = R.chunk_batch(ctx + B, 8, 2, D, 64, [ctx], [B], G.dev())
    pages = b["table"][0, first // 64:(first + keys) // 64].long()
    b["kp"][pages] = float("nan")
    assert bool(_run(b, CAUSAL).isnan().all())


@pytest.mark.parametrize("ctx", [[40, 90], [40, 9000]], ids=["one_launch", "planned"])
def test_a_context_below_zero_reads_nothing_before_its_table(ctx):
    """Lengths that the contract forbids: the sequence counts as one without a context, the other as it is."""
    b = R.chunk_batch(51, 16, 8, 128, 16, ctx, [70, 80], G.dev())
    most = max(ctx)
    b["ctx"][0] = -40
    got = _run(b, CAUSAL, max_ctx=most)
    b["ctx"][0] = 0
    R.assert_attended(got, b["q"], b["kp"], b["vp"], b["table"], b["ctx"], b["B"], b["off"], CAUSAL)
