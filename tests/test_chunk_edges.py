"""Single keys at the edges of steps, pieces and the causal mask of chunks over long contexts: their scores are six times
the others', so that leaving one out, or showing one too many, moves some row by more than its tolerance.  That this is so
is shown on the CPU, with the mistakes planted in the plain form; the kernel is then held to the same tolerance."""
import numpy as np
import pytest
import torch

import gpu_util as G
import paper_2606_31315_amd as sd
import prefill_ref as R

CTX, B, PAGE, PARTS = 20000, 100, 64, 8


def edge_keys(part):
    """First and last keys of every eighth step of 64, and the chunk's own keys."""
    steps = np.arange(part, (CTX + B) // 64, PARTS) * 64
    return np.concatenate([steps, steps + 63, np.arange(CTX, CTX + B)])


def edge_batch(D, part, device):
    b = R.chunk_batch(1000 + part, 8, 2, D, PAGE, [CTX, 0, 333], [B, 65, 1], "cpu")
    j = torch.from_numpy(np.unique(edge_keys(part)))
    pages, rows = b["table"][0].long()[j // PAGE], j % PAGE
    b["kp"][pages, :, rows] *= 6
    return {k: v.to(device) if isinstance(v, torch.Tensor) else v for k, v in b.items()}


def planted(q, k, v, hide=None, own=0):
    """The first sequence in 64 bits, without key `hide`, rows seeing `own` keys more (or fewer) than theirs."""
    Gq = q.shape[1] // k.shape[0]
    kd, vd = (x.double().repeat_interleave(Gq, 0) for x in (k, v))
    w = torch.matmul(q.double().transpose(0, 1), kd.transpose(1, 2)) * q.shape[2] ** -0.5
    w.masked_fill_(torch.arange(CTX + B) > CTX + own + torch.arange(B)[:, None], -np.inf)
    if hide is not None:
        w[..., hide] = -np.inf
    return torch.matmul(torch.softmax(w, -1), vd).transpose(0, 1)


@pytest.mark.parametrize("D", [64, 128])
def test_planted_mistakes_are_past_the_tolerance(D):
    b = edge_batch(D, 3, "cpu")
    k, v = (R.gathered(b[x], b["table"][0], CTX + B) for x in ("kp", "vp"))
    q, sound = b["q"][:B], (b["q"], b["kp"], b["vp"], b["table"], b["ctx"][:1], b["B"][:1], b["off"], R.CAUSAL)
    R.assert_attended(planted(q, k, v).to(torch.bfloat16), *sound)
    rng = np.random.default_rng(D)
    edges = edge_keys(3)
    edges = edges[edges < CTX]
    for kw in ([dict(own=1), dict(own=-1)] + [dict(hide=int(j)) for j in rng.choice(edges, 4, replace=False)] +
               [dict(hide=int(edges[0])), dict(hide=int(edges[-1]))]):
        with pytest.raises(AssertionError):
            R.assert_attended(planted(q, k, v, **kw).to(torch.bfloat16), *sound)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("part", range(PARTS))
def test_edges_of_cut_tiles(part, D):
    b = edge_batch(D, part, G.dev())
    lens = [torch.from_numpy(np.ascontiguousarray(b[x], np.int32)).to(G.dev()) for x in ("ctx", "B", "off")]
    G.log(f"sd_chunk_attn_paged, edge keys, part {part}, D={D}")
    o = sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], *lens, R.CAUSAL, max_ctx=CTX, max_chunk=B)
    torch.cuda.synchronize()
    R.assert_attended(o, b["q"], b["kp"], b["vp"], b["table"], b["ctx"], b["B"], b["off"], R.CAUSAL)
