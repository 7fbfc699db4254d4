"""Plain 64-bit forms of the operators that put a prompt into a paged cache, and the error that
their roundings allow.

Half a step of a type is U[type] relative to the value (bf16 2^-8, fp32 2^-24).

norm and rotation: everything between load and store is fp32, so an output differs from the exact one by
its own rounding, U |y|, and by the fp32 arithmetic before it, relative to the |a| + |b| of its pair:
at most 10 roundings in the mean square (halved by the root), 3 in root and weight, 4 in an
angle's sine (a turn rounded to fp32 times 2 pi, the sine itself), 3 in the rotation, below 2^-19
in all.

attention: the output's rounding, U |o|; the weights' rounding to bf16, U sum_j p_j |v_j| / l; and
fp32 sums, products and exponentials, whose share stays below 2^-12 of sum_j p_j |v_j| / l at the
tests' sizes (scores below 64 in size: 128 products 2^-24 each and one rounded exponent).
"""
import numpy as np
import torch

from paper_2606_31315_amd import workloads as W

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
CAUSAL, BIDIR = W.MASK_CAUSAL_IN_BLOCK, W.MASK_BIDIR_IN_BLOCK


def turned(x, w, pos, inv_freq, interleaved=False, eps=1e-6, rot_scale=1.0):
    """Norm (with a weight) and rotation of x [N, H, D] in 64 bits, and the size of each output's pair."""
    y = x.double().cpu()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double().cpu()
    size = y.abs()
    R = 0 if inv_freq is None else 2 * inv_freq.numel()
    if R:
        ang = pos.double().cpu()[:, None, None] * inv_freq.double().cpu()
        c, s = torch.cos(ang) * rot_scale, torch.sin(ang) * rot_scale
        ia = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
        ib = ia + (1 if interleaved else R // 2)
        a, b = y[..., ia], y[..., ib]
        out = y.clone()
        out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * max(1.0, abs(rot_scale))
        y = out
    return y, size


def assert_turned(got, ref, size):
    err = (got.double().cpu() - ref).abs()
    tol = U[got.dtype] * ref.abs() + 2.0 ** -19 * size
    bad = err > tol
    assert not bad.any(), (int(bad.sum()), float((err - tol).max()), bad.nonzero()[:3].tolist())


def attend(q, k, v, ctx, causal, scale=0.0):
    """Attention of one sequence in 64 bits: q [B, Hq, D], k and v [Hkv, ctx + B, D]; also the same with |v|."""
    B, Hq, D = q.shape
    G = Hq // k.shape[0]
    kd, vd = (x.double().repeat_interleave(G, 0) for x in (k, v))
    w = torch.matmul(q.double().transpose(0, 1).contiguous(), kd.transpose(1, 2).contiguous()) * (scale or D ** -0.5)
    if causal:
        w.masked_fill_(torch.arange(ctx + B, device=q.device) > ctx + torch.arange(B, device=q.device)[:, None], -np.inf)
    p = torch.softmax(w, -1)
    return torch.matmul(p, vd).transpose(0, 1), torch.matmul(p, vd.abs()).transpose(0, 1)


def gathered(pages, table, n):
    """The first n keys of a sequence, [Hkv, n, D], from a pool [num_pages, Hkv, page_size, D]."""
    ps = pages.shape[2]
    t = table[:-(-n // ps)].long()
    return pages[t].transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def assert_attended(got, q, k_pages, v_pages, table, ctx, B, off, mask, scale=0.0):
    """Every row of got against the plain form, sequence by sequence (on the inputs' device)."""
    for s in range(len(B)):
        if B[s] == 0:
            continue
        n, rows = int(ctx[s] + B[s]), slice(int(off[s]), int(off[s] + B[s]))
        ref, mag = attend(q[rows], gathered(k_pages, table[s], n), gathered(v_pages, table[s], n), int(ctx[s]),
                          mask == CAUSAL, scale)
        err = (got[rows].double() - ref).abs()
        tol = U[got.dtype] * ref.abs() + (U[torch.bfloat16] + 2.0 ** -12) * mag
        worst = float((err - tol).max())
        assert worst <= 0, (s, worst, float(err.max()), int((err > tol).sum()))


def chunk_batch(seed, Hq, Hkv, D, page, ctx, B, device, sigma=1.0, spare=3):
    """Queries, page pools and a shuffled block table of a ragged batch.  What no key of a sequence
    lies in (the rest of its last page, spare pages) is NaN."""
    g = torch.Generator().manual_seed(seed)
    ctx, B = np.asarray(ctx, np.int32), np.asarray(B, np.int32)
    off = W.offsets_from_lens(B)
    S, n = len(B), max(1, int(-(-(ctx + B).max() // page)))
    table = torch.randperm(S * n + spare, generator=g)[:S * n].reshape(S, n).to(torch.int32)
    q = (torch.randn(int(off[-1]), Hq, D, generator=g) * sigma).to(torch.bfloat16)
    kp, vp = (torch.full((S * n + spare, Hkv, page, D), float("nan"), dtype=torch.bfloat16) for _ in range(2))
    for s in range(S):
        L = int(ctx[s] + B[s])
        for x in (kp, vp):
            rows = torch.full((Hkv, n * page, D), float("nan"))
            rows[:, :L] = torch.randn(Hkv, L, D, generator=g)
            x[table[s].long()] = rows.reshape(Hkv, n, page, D).transpose(0, 1).to(torch.bfloat16)
    return dict(q=q.to(device), kp=kp.to(device), vp=vp.to(device), table=table.to(device), ctx=ctx, B=B, off=off)
