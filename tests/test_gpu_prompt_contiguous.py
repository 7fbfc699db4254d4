"""A prompt's way into the contiguous caches [S, Hkv, Lmax, D] of sd_block_attn and sd_verify_step: where Lmax is a page size
(a power of two from 16 to 4096), such a cache is a pool of one page per sequence, and the calls for pages fill it and attend
over it in place; any other is filled by sd_qk_norm_rope and sd_kv_append."""
import numpy as np
import pytest
import torch

import gpu_util as G
import paper_2606_31315_amd as sd
import prefill_ref as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(G.dev())


def _attended(o, q, kc, vc, ctx, B, off):
    """o against the plain form over the caches; fp32 weights are not rounded."""
    for s in range(len(B)):
        n, rows = int(ctx[s] + B[s]), slice(int(off[s]), int(off[s] + B[s]))
        ref, mag = R.attend(q[rows], kc[s, :, :n], vc[s, :, :n], int(ctx[s]), True)
        tol = R.U[o.dtype] * ref.abs() + ((R.U[BF] if o.dtype == BF else 0.0) + 2.0 ** -12) * mag
        assert float(((o[rows].double() - ref).abs() - tol).max()) <= 0, s


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("D,Lmax", [(128, 512), (64, 4096), (128, 256)])
def test_prompts_then_a_block(dt, D, Lmax):
    S, Hq, Hkv, dev = 3, 8, 2, G.dev()
    g = torch.Generator().manual_seed(D + Lmax)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dt).to(dev)  # noqa: E731
    P = np.array([Lmax - 30, 65, 1])
    off = np.concatenate([[0], np.cumsum(P)])
    x = rnd(int(off[-1]), (Hq + 2 * Hkv) * D)
    q, k, v = (t.unflatten(1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], 1))
    freq = (1e6 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(dev)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(dt).to(dev) for _ in range(2)]
    caches = [torch.full((S, Hkv, Lmax, D), 9.0, dtype=dt, device=dev) for _ in range(4)]
    kc, vc, k2, v2 = caches
    table, zero = torch.arange(S, dtype=torch.int32, device=dev)[:, None], _i32([0] * S)
    G.log(f"prompts into contiguous caches D={D} Lmax={Lmax} {dt}")
    # the caches as pages, and in two calls
    qr = sd.kv_append_rope_paged(q, k, v, kc, vc, table, zero, _i32(off), freq, q_weight=w[0], k_weight=w[1])
    pos = _i32(np.concatenate([np.arange(n) for n in P]))
    q2, kr = sd.qk_norm_rope(q, k, pos, freq, q_weight=w[0], k_weight=w[1])
    sd.kv_append(kr, v.contiguous(), k2, v2, zero, _i32(off))
    torch.cuda.synchronize()
    assert torch.equal(qr, q2) and torch.equal(kc, k2) and torch.equal(vc, v2)
    assert all(bool((c[s, :, P[s]:] == 9.0).all()) for c in caches for s in range(S))
    if dt == BF:
        o = sd.chunk_attn_paged(qr, kc, vc, table, zero, _i32(P), _i32(off), R.CAUSAL, max_ctx=0, max_chunk=int(P.max()))
        torch.cuda.synchronize()
        _attended(o, qr, kc, vc, [0] * S, P, off)
    # a block over the same caches
    B = np.array([16, 1, 7])
    boff = np.concatenate([[0], np.cumsum(B)])
    n = int(boff[-1])
    qb, kb, vb = rnd(n, Hq, D), rnd(n, Hkv, D), rnd(n, Hkv, D)
    sd.kv_append(kb, vb, kc, vc, _i32(P), _i32(boff))
    o = sd.block_attn(qb, kc, vc, _i32(P), _i32(B), _i32(boff), R.CAUSAL, max_ctx=int(P.max()), max_block=16)
    torch.cuda.synchronize()
    _attended(o, qb, kc, vc, P, B, boff)
