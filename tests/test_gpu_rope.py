"""sd_qk_norm_rope and sd_kv_append_rope_paged against the plain form in 64 bits, and the way of a
prompt through them: append, chunk attention, then a block's verification over the same pages."""
import numpy as np
import pytest
import torch

import gpu_util as G
import oracle.paged as OPG
import paper_2606_31315_amd as sd
import prefill_ref as R
from paper_2606_31315_amd import workloads as W

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(G.dev())


def _inv_freq(R_, theta=1e6):
    return (theta ** (-torch.arange(0, R_, 2, dtype=torch.float64) / R_)).float().to(G.dev()) if R_ else None


def _packed(seed, N, Hq, Hkv, D, dt, pad=0):
    """q, k, v as slices of one projection's rows (pad: elements between them and the next row)."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, (Hq + 2 * Hkv) * D + pad, generator=g) * torch.exp(torch.randn(N, 1, generator=g))).to(dt).to(G.dev())
    q, k, v = x[:, :Hq * D], x[:, Hq * D:(Hq + Hkv) * D], x[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D]
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


def _weights(seed, D, dt):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.2 * torch.randn(D, generator=g)).to(dt).to(G.dev()) for _ in range(2)]


ROPE = [  # rows, Hq, Hkv, D, rotated dims, interleaved, norm, dtype, pad, furthest position
    (1, 32, 8, 128, 128, False, True, BF, 0, 40960),
    (7, 32, 8, 128, 128, False, True, BF, 8, 1 << 30),
    (130, 32, 4, 128, 64, True, True, BF, 0, 4096),
    (33, 16, 8, 64, 64, False, True, F32, 4, 100000),
    (65, 5, 1, 64, 48, False, False, F32, 0, 1 << 20),
    (64, 3, 3, 128, 16, True, False, BF, 0, 1000),
    (9, 8, 8, 128, 112, False, True, F32, 12, 1 << 24),
    (3, 17, 2, 64, 0, False, True, BF, 0, 10),
    (2000, 8, 2, 64, 64, True, True, BF, 0, 131072),
]


@pytest.mark.parametrize("N,Hq,Hkv,D,rot,inter,norm,dt,pad,far", ROPE)
def test_qk_norm_rope(N, Hq, Hkv, D, rot, inter, norm, dt, pad, far):
    q, k, _ = _packed(N, N, Hq, Hkv, D, dt, pad)
    pos = torch.randint(0, far, (N,), generator=torch.Generator().manual_seed(N), dtype=torch.int32)
    pos[0] = far - 1
    qw, kw = _weights(N, D, dt) if norm else (None, None)
    f = _inv_freq(rot)
    G.log(f"sd_qk_norm_rope N={N} Hq={Hq} Hkv={Hkv} D={D} rot={rot} inter={inter} norm={norm} dtype={dt}")
    qo, ko = sd.qk_norm_rope(q, k, pos.to(G.dev()), f, q_weight=qw, k_weight=kw, interleaved=inter)
    torch.cuda.synchronize()
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        R.assert_turned(got, *R.turned(x, w, pos, f, inter))


def test_in_place_one_side_and_negative_positions():
    q, k, _ = _packed(3, 21, 8, 2, 128, BF)
    pos = torch.arange(-10, 11, dtype=torch.int32)
    f = _inv_freq(128)
    qw, kw = _weights(3, 128, BF)
    rq, rk = R.turned(q, qw, pos, f), R.turned(k, None, pos, f, rot_scale=1.25)
    v = torch.empty_like(k)
    G.log("sd_qk_norm_rope in place")
    o, none = sd.qk_norm_rope(q, None, pos.to(G.dev()), f, q_weight=qw, q_out=q)
    assert none is None and o is q
    none, o = sd.qk_norm_rope(None, k, pos.to(G.dev()), f, rot_scale=1.25, k_out=v)
    assert none is None and o is v
    torch.cuda.synchronize()
    R.assert_turned(q, *rq)
    R.assert_turned(v, *rk)


@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-2])
def test_small_and_zero_rows(eps):
    """eps decides for heads near zero; a zero head stays zero with one."""
    q = torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(1))
    q[1], q[2] = q[1] * 1e-3, 0.0
    if eps == 0.0:
        q[2] = 1.0
    q = q.to(BF).to(G.dev())
    w = _weights(1, 128, BF)[0]
    pos = torch.arange(4, dtype=torch.int32)
    G.log(f"sd_qk_norm_rope eps={eps}")
    o, _ = sd.qk_norm_rope(q, None, pos.to(G.dev()), _inv_freq(128), q_weight=w, eps=eps)
    R.assert_turned(o, *R.turned(q, w, pos, _inv_freq(128), eps=eps))


def test_non_finite_heads_stay_apart():
    """An infinity or NaN in one head reaches that head only."""
    q, k, _ = _packed(5, 6, 16, 8, 128, BF)
    pos, f, (qw, kw) = _i32(np.arange(6)), _inv_freq(128), _weights(5, 128, BF)
    ref, refk = sd.qk_norm_rope(q, k, pos, f, q_weight=qw, k_weight=kw)
    q[2, 3, 7], q[4, 9, 100] = float("nan"), float("inf")
    got, gotk = sd.qk_norm_rope(q, k, pos, f, q_weight=qw, k_weight=kw)
    torch.cuda.synchronize()
    keep = torch.ones(6, 16, dtype=torch.bool, device=G.dev())
    keep[2, 3] = keep[4, 9] = False
    assert torch.equal(got[keep], ref[keep]) and torch.equal(gotk, refk)
    assert bool(got[2, 3].isnan().all()) and bool(got[4, 9].isnan().any())


APPEND = [  # Hq, Hkv, D, page, rot, interleaved, norm, dtype, contexts, rows
    (32, 8, 128, 16, 128, False, True, BF, [100, 0, 250], [16, 1, 70]),
    (32, 8, 128, 64, 128, False, True, BF, [511, 64, 3], [1, 1, 1]),
    (8, 8, 64, 256, 32, True, False, F32, [90000, 255], [3, 2]),
    (16, 2, 64, 32, 64, False, True, BF, [31, 32, 0, 5], [0, 129, 33, 0]),
    (0, 4, 128, 16, 128, False, True, BF, [7, 77], [20, 9]),
    (6, 3, 128, 16, 0, False, False, F32, [0], [300]),
]


@pytest.mark.parametrize("Hq,Hkv,D,page,rot,inter,norm,dt,ctx,B", APPEND)
def test_append(Hq, Hkv, D, page, rot, inter, norm, dt, ctx, B):
    """Keys normed and rotated at their places in the pages, values as they were, everything else untouched."""
    dev, off = G.dev(), W.offsets_from_lens(np.array(B, np.int32))
    N, S, n = int(off[-1]), len(B), max(-(-(c + b) // page) for c, b in zip(ctx, B))
    q, k, v = _packed(N, N, max(Hq, 1), Hkv, D, dt)
    q = q if Hq else None
    g = torch.Generator().manual_seed(N)
    table = torch.randperm(S * n + 3, generator=g)[:S * n].reshape(S, n).to(torch.int32)
    kp, vp = (torch.randn(S * n + 3, Hkv, page, D, generator=g).to(dt) for _ in range(2))
    dkp, dvp = kp.to(dev), vp.to(dev)
    qw, kw = _weights(N, D, dt) if norm else (None, None)
    f = _inv_freq(rot)
    G.log(f"sd_kv_append_rope_paged N={N} Hq={Hq} Hkv={Hkv} D={D} page={page} rot={rot} dtype={dt}")
    qo = sd.kv_append_rope_paged(q, k, v, dkp, dvp, table.to(dev), _i32(ctx), _i32(off), f,
                                 q_weight=qw if Hq else None, k_weight=kw, interleaved=inter)
    torch.cuda.synchronize()
    pos = torch.cat([c + torch.arange(b) for c, b in zip(ctx, B)])
    if Hq:
        R.assert_turned(qo, *R.turned(q, qw, pos, f, inter))
    else:
        assert qo is None
    # the keys against the plain form, then put into the plain append: everything else has to be equal
    seq = np.repeat(np.arange(S), B)
    page_of, at = table[seq, pos // page].long(), pos % page
    R.assert_turned(dkp.cpu()[page_of, :, at], *R.turned(k, kw, pos, f, inter))
    rk, rv = OPG.kv_append_paged(kp, vp, table.numpy(), dkp.cpu()[page_of, :, at], v, ctx, off)
    assert np.array_equal(dkp.float().cpu().numpy(), rk) and np.array_equal(dvp.float().cpu().numpy(), rv)


def test_append_skips_what_has_no_page_and_padding():
    """Rows past the table or with a page id outside the pool are not written; rows behind the last
    sequence change nothing; their queries' places neither."""
    dev, page, Hkv, D = G.dev(), 16, 2, 128
    ctx, B = np.array([40, 10], np.int32), np.array([20, 30], np.int32)  # sequence 0: 48 keys in the table
    off = W.offsets_from_lens(B)
    q, k, v = _packed(8, 57, 4, Hkv, D, BF)
    table = torch.tensor([[4, 0, 7], [1, 9000, 2]], dtype=torch.int32)
    table2 = table.clone()
    table2[1, 1] = -1
    g = torch.Generator().manual_seed(8)
    kp, vp = (torch.randn(9, Hkv, page, D, generator=g).to(BF) for _ in range(2))
    f = _inv_freq(128)
    for t in (table, table2):
        dkp, dvp, qo = kp.to(dev), vp.to(dev), torch.full((57, 4, D), 5.0, dtype=BF, device=dev)
        G.log("sd_kv_append_rope_paged past the table, bad ids, padding")
        sd.kv_append_rope_paged(q, k, v, dkp, dvp, t.to(dev), _i32(ctx), _i32(off), f, q_out=qo)
        torch.cuda.synchronize()
        assert bool((qo[50:] == 5.0).all())
        pos = torch.cat([c + torch.arange(int(b)) for c, b in zip(ctx, B)])
        R.assert_turned(qo[:50], *R.turned(q[:50], None, pos, f))
        ko, _ = sd.qk_norm_rope(k[:50], None, pos.to(torch.int32).to(dev), f)
        rk, rv = OPG.kv_append_paged(kp, vp, t.numpy(), ko, v, ctx, off)
        assert np.array_equal(dkp.float().cpu().numpy(), rk) and np.array_equal(dvp.float().cpu().numpy(), rv)


def test_append_many_sequences_matches_the_two_steps():
    """150 sequences, empty ones among them: the same bits as sd_qk_norm_rope and sd_kv_append_paged."""
    rng = np.random.default_rng(2)
    dev, B, ctx = G.dev(), rng.integers(0, 9, 150).astype(np.int32), rng.integers(0, 90, 150).astype(np.int32)
    B[[0, 63, 64, 65, 128, 149]] = 0
    off = W.offsets_from_lens(B)
    q, k, v = _packed(9, int(off[-1]), 8, 4, 128, BF)
    table = torch.randperm(150 * 7, generator=torch.Generator().manual_seed(1)).reshape(150, 7).to(torch.int32).to(dev)
    kp, vp, kp2, vp2 = (torch.zeros(150 * 7, 4, 16, 128, dtype=BF, device=dev) for _ in range(4))
    qw, kw = _weights(9, 128, BF)
    f = _inv_freq(128)
    G.log("sd_kv_append_rope_paged S=150")
    qo = sd.kv_append_rope_paged(q, k, v, kp, vp, table, _i32(ctx), _i32(off), f, q_weight=qw, k_weight=kw)
    pos = _i32(np.concatenate([c + np.arange(b) for c, b in zip(ctx, B)]))
    q2, k2 = sd.qk_norm_rope(q, k, pos, f, q_weight=qw, k_weight=kw)
    sd.kv_append_paged(k2, v.contiguous(), kp2, vp2, table, _i32(ctx), _i32(off))
    torch.cuda.synchronize()
    assert torch.equal(qo, q2) and torch.equal(kp, kp2) and torch.equal(vp, vp2)


def test_append_pools_past_32_bit_offsets():
    dev, page, Hkv, D = G.dev(), 256, 8, 128
    n = (1 << 31) // (Hkv * page * D) + 5
    kp, vp = (torch.empty(n, Hkv, page, D, dtype=BF, device=dev) for _ in range(2))
    table = torch.tensor([[n - 1, 0, n - 2]], dtype=torch.int32, device=dev)
    kp[table[0].long()], vp[table[0].long()] = 0.0, 0.0
    q, k, v = _packed(4, 600, 4, Hkv, D, BF)
    G.log("sd_kv_append_rope_paged past 2^31 elements")
    sd.kv_append_rope_paged(None, k, v, kp, vp, table, _i32([100]), _i32([0, 600]), _inv_freq(128))
    torch.cuda.synchronize()
    at = 100 + torch.arange(600, device=dev)
    page_of = table[0, at // page].long()
    R.assert_turned(kp[page_of, :, at % page], *R.turned(k, None, at, _inv_freq(128)))
    assert torch.equal(vp[page_of, :, at % page], v)


@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 32, 8, 16), (64, 8, 4, 64)])
def test_a_prompt_through_the_cache(D, Hq, Hkv, page):
    """Two prompts in chunks of different lengths, then a drafted block: append and attention of every chunk, the
    block's verification by the block attention, all against attention over the exact keys of the pages."""
    dev, S, n = G.dev(), 2, 600
    f = _inv_freq(D)
    qw, kw = _weights(D, D, BF)
    kp, vp = (torch.full((2 * (n // page + 1) + 1, Hkv, page, D), float("nan"), dtype=BF, device=dev) for _ in range(2))
    table = torch.randperm(kp.shape[0] - 1, generator=torch.Generator().manual_seed(D))[:2 * (n // page)]
    table = table.reshape(2, -1).to(torch.int32).to(dev)
    ctx = np.zeros(2, np.int32)
    for step, B in enumerate(([300, 1], [0, 257], [131, 90], [1, 1], [16, 12])):
        B = np.array(B, np.int32)
        off = W.offsets_from_lens(B)
        q, k, v = _packed(100 + step, int(off[-1]), Hq, Hkv, D, BF)
        G.log(f"prompt step {step}: ctx {ctx.tolist()} rows {B.tolist()}")
        qo = sd.kv_append_rope_paged(q, k, v, kp, vp, table, _i32(ctx), _i32(off), f, q_weight=qw, k_weight=kw)
        call = sd.chunk_attn_paged if step < 4 else sd.block_attn_paged
        bound = {"max_chunk" if step < 4 else "max_block": int(B.max())}
        o = call(qo, kp, vp, table, _i32(ctx), _i32(B), _i32(off), R.CAUSAL, max_ctx=int(ctx.max()), **bound)
        torch.cuda.synchronize()
        R.assert_attended(o, qo, kp, vp, table, ctx, B, off, R.CAUSAL)
        ctx += B


def test_graph_replays():
    """Captured once, replayed while positions advance: the same pages as eager calls."""
    dev = G.dev()
    q, k, v = _packed(6, 3, 8, 4, 128, BF)
    f = _inv_freq(128)
    table = torch.arange(3 * 4, dtype=torch.int32, device=dev).reshape(3, 4)
    pools = {x: [torch.zeros(12, 4, 16, 128, dtype=BF, device=dev) for _ in range(2)] + [torch.zeros_like(q)]
             for x in ("graph", "eager")}
    ctx, off = _i32([0, 15, 30]), _i32([0, 1, 2, 3])

    def call(x):
        sd.kv_append_rope_paged(q, k, v, *pools[x][:2], table, ctx, off, f, q_out=pools[x][2])

    call("eager")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call("graph")
    for i in range(5):
        call("eager")
        graph.replay()
        torch.cuda.synchronize()
        if i == 0:  # the eager call before the capture wrote the same places
            pass
        assert all(torch.equal(a, b) for a, b in zip(pools["graph"], pools["eager"])), i
        ctx += 1
        q.mul_(1.5), k.mul_(-0.75), v.add_(1.0)
        torch.cuda.synchronize()


def test_more_rows_than_workgroups():
    """4.3 million rows of one head: the grid ends at 2^20 workgroups, which go round."""
    N = 4_300_000
    q = torch.randn(N, 1, 64, dtype=BF, device=G.dev())
    pos = torch.arange(N, dtype=torch.int32, device=G.dev())
    f = _inv_freq(64)
    G.log(f"sd_qk_norm_rope N={N}")
    o, _ = sd.qk_norm_rope(q, None, pos, f)
    torch.cuda.synchronize()
    for lo in (0, (1 << 22) - 8, N - 16):
        R.assert_turned(o[lo:lo + 16], *R.turned(q[lo:lo + 16], None, pos[lo:lo + 16], f))
