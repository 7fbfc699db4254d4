"""Performance cases of the operators that put a prompt's tokens into a paged cache and attend over it:
norm and rotation of queries and keys, the append that does both on the way into the pages, and the
attention of chunks of new tokens.

A case is a dict of plain values.  `listed()` are the named cases, `draw()` makes more of the same
ranges, `prepare()` builds what a caller holds before the call (on the GPU), `run()` is one pass,
`work()` the bytes and operations a pass cannot do without and `exact()` the same outputs in 64 bits.
With `own` false `run()` computes the operators by elementary torch operations in 32 bits (angles in
64), rounded once at the end; with `own` true it makes the library's calls.

Ragged lengths follow from the case alone (`lens` seeds them), so the work of a case is known without
its inputs; values follow from the seed given to `prepare()`.
"""
import math
import random

import torch

own = False  # run(): the library's kernels instead of the plain form

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
THETA = 1e6  # base of the rotation's frequencies


def _rope(name, N, heads=(32, 8), D=128, dtype="bf16", rot=None, inter=False, norm=True, far=40960):
    return {"name": name, "op": "rope", "N": N, "Hq": heads[0], "Hkv": heads[1], "D": D, "dtype": dtype,
            "rot": D if rot is None else rot, "inter": inter, "norm": norm, "far": far}


def _append(name, S, ctx, rows, page, heads=(32, 8), D=128, dtype="bf16", rot=None, inter=False, norm=True, lens=1):
    return {"name": name, "op": "append", "S": S, "Hq": heads[0], "Hkv": heads[1], "D": D, "dtype": dtype,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "b_lo": rows[0], "b_hi": rows[1], "ones": 0.0, "page": page,
            "rot": D if rot is None else rot, "inter": inter, "norm": norm, "lens": lens}


def _chunk(name, S, ctx, rows, page, heads=(32, 8), D=128, mask="causal", ones=0.0, lens=1):
    return {"name": name, "op": "chunk", "S": S, "Hq": heads[0], "Hkv": heads[1], "D": D, "dtype": "bf16",
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "b_lo": rows[0], "b_hi": rows[1], "ones": ones, "page": page,
            "mask": mask, "lens": lens}


def listed():
    return [
        # one token of one sequence in one layer: the smallest call, all latency
        _rope("rope_token_b1", 1),
        # a prompt of 8192 tokens, queries, keys and values in one projection's rows
        _rope("rope_prompt_8k", 8192),
        # a model kept in fp32: half of each head rotated, neighbouring pairs, an odd number of rows
        _rope("rope_fp32_odd", 1537, heads=(16, 8), D=64, dtype="f32", rot=32, inter=True),
        # a decoding batch: one token of each of 32 sequences goes to its page
        _append("append_decode_b32", 32, (500, 4000), (1, 1), 64, lens=2),
        # prompt chunks of four sequences, small pages
        _append("append_prompt_b4", 4, (0, 6000), (1000, 2048), 16, lens=3),
        # fp32 pages far into long contexts, no norm, a few odd rows
        _append("append_fp32_far", 3, (60000, 100000), (5, 77), 256, heads=(8, 8), D=64, dtype="f32", norm=False,
                lens=4),
        # the tail of a prompt: a short chunk over a short context
        _chunk("chunk_tail_b1", 1, (500, 500), (100, 100), 64),
        # a whole prompt in one chunk
        _chunk("chunk_prompt_8k", 1, (0, 0), (8192, 8192), 64),
        # several prompts at different places of their chunks, odd lengths
        _chunk("chunk_ragged_b8", 8, (0, 6001), (200, 1501), 16, lens=6),
        # a serving batch: prompt chunks of some sequences beside single tokens of the others
        _chunk("chunk_mixed_b32", 32, (1000, 16000), (500, 2000), 64, ones=0.8, lens=7),
        # a chunk late in a long context, eight query heads to a kv head
        _chunk("chunk_long_64k", 1, (65536, 65536), (2048, 2048), 256, heads=(32, 4)),
        # the block-diffusion drafter over a prompt: bidirectional, small heads, one kv head to a query head
        _chunk("chunk_bidir_d64", 4, (300, 3001), (300, 1201), 32, heads=(8, 8), D=64, mask="bidir", lens=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: one row to 8192, contexts from none to 64k, both head sizes, masks,
    pair orders and types, pages of 16 to 256 keys."""
    op = rng.choice(["rope", "append", "chunk", "chunk"])
    heads, D = rng.choice([(32, 8), (32, 8), (32, 4), (16, 8), (8, 8)]), rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rot = rng.choice([D, D, D // 2, 48])
    kw = {"dtype": dtype, "rot": rot, "inter": rng.random() < 0.3, "norm": rng.random() < 0.7}
    lens = rng.randrange(1 << 20)
    page = rng.choice([16, 32, 64, 256])
    if op == "rope":
        c = _rope("", _log(rng, 1, 8192), heads, D, far=_log(rng, 100, 1 << 20), **kw)
    elif op == "append":
        S = _log(rng, 1, 32)
        hi = _log(rng, 1, max(2, 8192 // S))
        top = _log(rng, 100, max(200, 120_000 // S))
        c = _append("", S, (int(top * rng.random()), top), (max(1, int(hi * rng.random())), hi), page, heads, D,
                    lens=lens, **kw)
    else:
        S = _log(rng, 1, 32)
        hi = _log(rng, 2, max(3, 8192 // S))
        top = _log(rng, 20, max(30, min(65536, 500_000 // max(S, hi // 8))))
        c = _chunk("", S, (int(top * rng.random()), top), (max(1, int(hi * rng.random())), hi), page, heads, D,
                   rng.choice(["causal", "causal", "bidir"]), rng.choice([0.0, 0.0, 0.7]), lens)
    c.pop("name")
    return c


def _lens(case):
    """Contexts, rows and row offsets of the sequences; a share `ones` of them brings a single row."""
    r = random.Random(case["lens"])
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["S"])]
    blk = [r.randint(case["b_lo"], case["b_hi"]) for _ in range(case["S"])]
    blk = [1 if i and r.random() < case["ones"] else b for i, b in enumerate(blk)]
    off = [0]
    for b in blk:
        off.append(off[-1] + b)
    return ctx, blk, off


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


# ---- what a caller holds ----

def _projected(case, g, n, dt):
    """Rows of one projection: queries, keys and values side by side, so each is a strided view."""
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    qkv = _randn(g, (n, (Hq + 2 * Hkv) * D), dt)
    q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], 1)
    st = {"q": q.view(n, Hq, D), "k": k.view(n, Hkv, D), "v": v.view(n, Hkv, D), "inter": case["inter"]}
    i = torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64)
    st["inv_freq"] = (THETA ** (-i / case["rot"])).float()
    st["qw"] = st["kw"] = None
    if case["norm"]:
        st["qw"], st["kw"] = ((1 + 0.1 * _randn(g, (D,), torch.float32)).to(dt) for _ in range(2))
    return st


def _pool(case, seed, g, dt, L):
    """Page pools with three pages to spare and a shuffled block table."""
    ps, S = case["page"], case["S"]
    n = -(-L // ps)
    pool = S * n + 3
    perm = torch.randperm(pool, generator=torch.Generator().manual_seed(seed))[:S * n]
    shape = (pool, case["Hkv"], ps, case["D"])
    return {"table": perm.to(torch.int32).reshape(S, n).to(DEV), "kp": _randn(g, shape, dt),
            "vp": _randn(g, shape, dt)}


def prepare(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    if case["op"] == "rope":
        st = _projected(case, g, case["N"], dt)
        st["pos"] = torch.randint(0, case["far"], (case["N"],), generator=g, device=DEV, dtype=torch.int32)
        st["q_out"] = torch.empty(st["q"].shape, dtype=dt, device=DEV)
        st["k_out"] = torch.empty(st["k"].shape, dtype=dt, device=DEV)
    else:
        ctx, blk, off = _lens(case)
        st = _pool(case, seed, g, dt, max(c + b for c, b in zip(ctx, blk)))
        if case["op"] == "append":
            st.update(_projected(case, g, off[-1], dt))
            st["q_out"] = torch.empty(st["q"].shape, dtype=dt, device=DEV)
        else:
            st.update(q=_randn(g, (off[-1], case["Hq"], case["D"]), dt), blk=_i32(blk), causal=case["mask"] == "causal",
                      max_ctx=max(ctx), max_chunk=max(blk))
            st["out"] = torch.empty_like(st["q"])
        st.update(ctx=_i32(ctx), off=_i32(off), lens=(ctx, blk, off))
    st["op"] = case["op"]
    return st


# ---- the plain forms ----

def _turned(x, w, pos, st):
    """Norm over each head (with a weight) and rotation, in 32 bits from 64-bit angles; one rounding at the end."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.float()
    ang = pos.double()[:, None, None] * st["inv_freq"].double()
    c, s = torch.cos(ang).float(), torch.sin(ang).float()
    R = 2 * c.shape[-1]
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if st["inter"] else (y[..., :R // 2], y[..., R // 2:R])
    ya, yb = a * c - b * s, b * c + a * s
    turned = torch.stack((ya, yb), -1).flatten(-2) if st["inter"] else torch.cat((ya, yb), -1)
    return torch.cat((turned, y[..., R:]), -1).to(x.dtype)


def _run_append(st):
    rows = torch.arange(st["q"].shape[0], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["off"], rows, right=True) - 1
    pos = st["ctx"][seq] + rows - st["off"][seq]
    ps = st["kp"].shape[2]
    page = st["table"][seq, (pos // ps).long()].long()
    at = (pos % ps).long()
    st["q_out"].copy_(_turned(st["q"], st["qw"], pos, st))
    st["kp"][page, :, at] = _turned(st["k"], st["kw"], pos, st)
    st["vp"][page, :, at] = st["v"]
    return {"q": st["q_out"], "k_pages": st["kp"], "v_pages": st["vp"]}


def _run_chunk(st):
    """Sequence by sequence, 1024 positions at a time: scores, softmax and weighted values in 32 bits."""
    ctx, blk, off = st["lens"]
    Hq, D = st["q"].shape[1:]
    _, Hkv, ps, _ = st["kp"].shape
    G = Hq // Hkv
    for s, (c, b) in enumerate(zip(ctx, blk)):
        t = st["table"][s, :-(-(c + b) // ps)]
        k, v = (x[t].transpose(0, 1).reshape(Hkv, -1, D)[:, :c + b].float() for x in (st["kp"], st["vp"]))
        kt = k.transpose(1, 2).contiguous()
        for i in range(0, b, 1024):
            n = min(1024, b - i)
            L = c + i + n if st["causal"] else c + b
            q = st["q"][off[s] + i:off[s] + i + n].float().reshape(n, Hkv, G, D).permute(1, 2, 0, 3)
            w = torch.matmul(q.reshape(Hkv, G * n, D), kt[:, :, :L].contiguous()).div_(math.sqrt(D))
            if st["causal"]:
                hide = torch.arange(L, device=DEV)[None] > c + i + torch.arange(n, device=DEV)[:, None]
                w.view(Hkv, G, n, L).masked_fill_(hide, float("-inf"))
            w = w.sub_(w.amax(-1, keepdim=True)).exp_()
            o = torch.matmul(w, v[:, :L].contiguous()) / w.sum(-1, keepdim=True)
            st["out"][off[s] + i:off[s] + i + n] = o.view(Hkv, G, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D).to(st["q"].dtype)
    return st["out"]


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "rope":
        st["q_out"].copy_(_turned(st["q"], st["qw"], st["pos"], st))
        st["k_out"].copy_(_turned(st["k"], st["kw"], st["pos"], st))
        return {"q": st["q_out"], "k": st["k_out"]}
    return _run_append(st) if st["op"] == "append" else _run_chunk(st)


# ---- the library's calls ----

def _run_own(st):
    import paper_2606_31315_amd as sd
    if st["op"] == "rope":
        q, k = sd.qk_norm_rope(st["q"], st["k"], st["pos"], st["inv_freq"], q_weight=st["qw"], k_weight=st["kw"],
                               eps=EPS, interleaved=st["inter"], q_out=st["q_out"], k_out=st["k_out"])
        return {"q": q, "k": k}
    if st["op"] == "append":
        q = sd.kv_append_rope_paged(st["q"], st["k"], st["v"], st["kp"], st["vp"], st["table"], st["ctx"], st["off"],
                                    st["inv_freq"], q_weight=st["qw"], k_weight=st["kw"], eps=EPS,
                                    interleaved=st["inter"], q_out=st["q_out"])
        return {"q": q, "k_pages": st["kp"], "v_pages": st["vp"]}
    mask = sd.SD_MASK_CAUSAL_IN_BLOCK if st["causal"] else sd.SD_MASK_BIDIR_IN_BLOCK
    return sd.chunk_attn_paged(st["q"], st["kp"], st["vp"], st["table"], st["ctx"], st["blk"], st["off"], mask,
                               max_ctx=st["max_ctx"], max_chunk=st["max_chunk"], out=st["out"])


# ---- work and exact results ----

def work(case):
    Hq, Hkv, D, e = case["Hq"], case["Hkv"], case["D"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        n = case["N"]
        return {"bytes": n * ((Hq + Hkv) * D * e * 2 + 4) + 2 * case["rot"], "flops": n * (Hq + Hkv) * D * 8}
    ctx, blk, off = _lens(case)
    n, S = off[-1], case["S"]
    if case["op"] == "append":
        return {"bytes": n * ((Hq + 2 * Hkv) * D * e * 2 + 4) + 8 * S + 2 * case["rot"], "flops": n * (Hq + Hkv) * D * 8}
    keys = sum(c + b for c, b in zip(ctx, blk))
    causal = case["mask"] == "causal"
    pairs = sum(b * c + (b * (b + 1) // 2 if causal else b * b) for c, b in zip(ctx, blk))
    return {"bytes": 2 * n * Hq * D * e + 2 * keys * Hkv * D * e + 4 * keys // case["page"], "flops": 4 * D * Hq * pairs}


def _exact_turned(x, w, pos, freq, case):
    """The norm and the rotation as a product of complex numbers, in 64 bits."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).sum(2, keepdim=True) / y.shape[2] + EPS) * w.double()
    R = case["rot"]
    e = torch.outer(pos.double(), freq.double())[:, None]
    e = torch.polar(torch.ones_like(e), e)
    out = y.clone()
    even = slice(0, R, 2) if case["inter"] else slice(0, R // 2)
    odd = slice(1, R, 2) if case["inter"] else slice(R // 2, R)
    z = torch.complex(y[:, :, even], y[:, :, odd]) * e
    out[:, :, even], out[:, :, odd] = z.real, z.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return {x: _exact_turned(st[x], st[w], st["pos"], st["inv_freq"], case) for x, w in (("q", "qw"), ("k", "kw"))}
    ctx, blk, off = _lens(case)
    ps, Hkv, D = case["page"], case["Hkv"], case["D"]
    if case["op"] == "append":
        pos = torch.cat([c + torch.arange(b, device=DEV) for c, b in zip(ctx, blk)])
        k, kp, vp = _exact_turned(st["k"], st["kw"], pos, st["inv_freq"], case), st["kp"].double(), st["vp"].double()
        table = st["table"].tolist()
        for s, (c, b) in enumerate(zip(ctx, blk)):
            for j in range(c // ps, (c + b - 1) // ps + 1):  # the part of the rows that lies in logical page j
                lo, hi = max(c, j * ps), min(c + b, (j + 1) * ps)
                r = slice(off[s] + lo - c, off[s] + hi - c)
                kp[table[s][j], :, lo - j * ps:hi - j * ps] = k[r].transpose(0, 1)
                vp[table[s][j], :, lo - j * ps:hi - j * ps] = st["v"][r].transpose(0, 1).double()
        return {"q": _exact_turned(st["q"], st["qw"], pos, st["inv_freq"], case), "k_pages": kp, "v_pages": vp}
    G = case["Hq"] // Hkv
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    for s, (c, b) in enumerate(zip(ctx, blk)):
        key = torch.arange(c + b, device=DEV)
        page, at = st["table"][s].long()[key // ps], key % ps
        for h in range(Hkv):
            k, v = st["kp"][page, h, at].double(), st["vp"][page, h, at].double()
            for i in range(0, b, 512):
                n = min(512, b - i)
                q = st["q"][off[s] + i:off[s] + i + n, h * G:(h + 1) * G].double()
                w = (q.reshape(n * G, D) @ k.t().contiguous()).view(n, G, -1) * D ** -0.5
                if case["mask"] == "causal":
                    w.masked_fill_((key[None] > c + i + torch.arange(n, device=DEV)[:, None])[:, None], -math.inf)
                out[off[s] + i:off[s] + i + n, h * G:(h + 1) * G] = (torch.softmax(w, 2).view(n * G, -1) @ v).view(n, G, D)
    return out
